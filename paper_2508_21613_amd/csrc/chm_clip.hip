// Global norm of a list of gradients, and clipping by it.
//
// norm^2 = sum g^2 over all tensors, out = g min(1, max_norm / (norm + 1e-6)).  Both passes do nothing but move bytes: N are read for
// the norm, N read and N written for the clipping (in place and within the norm, nothing is written).  The tensors are cut into
// pieces of 16 KiB, which workgroups take in runs: one launch for each pass however many tensors there are, a workgroup's first
// piece is looked up in a table made at load.  Squares are summed in float64: those of float32 values neither overflow nor vanish
// there, and the additions hide behind the loads.  The second launch's workgroups each add up the first one's sums (at most
// 2,048, in one fixed order), which costs less than a launch between the two.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <new>
#include <vector>

#include "chm_elements.h"

namespace {

using namespace chm_elements;

constexpr int PIECE = 16384;             // bytes
constexpr int GROUPS_MAX = 2048;         // 8 workgroups of 256 for each of 256 CUs
constexpr int NT = 256;

struct Tensor { const char *in; char *out; int64_t n; int32_t dtype; int32_t bytes; };
struct Start { int32_t tensor; int32_t piece; };       // first tensor of a workgroup's run, first piece within it

struct List {
  const Tensor *tensors;
  const Start *starts;
  int32_t count, groups;
  int64_t pieces;
};

// One piece: `bytes` of a tensor from p on; adds its squares up
template <int DT, int THREADS>
__device__ __forceinline__ double piece_sum(const char *p, int bytes) {
  typedef Lane<DT> L;
  double s0 = 0, s1 = 0;
  constexpr int PER = PIECE / 16 / THREADS > 0 ? PIECE / 16 / THREADS : 1;
  if (bytes == PIECE) {
    Words x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = load16(p + (i * THREADS + threadIdx.x) * 16);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float v[8];
      L::up(x[i], v);
#pragma unroll
      for (int e = 0; e < L::N; e += 2) { s0 = fma((double)v[e], (double)v[e], s0); s1 = fma((double)v[e + 1], (double)v[e + 1], s1); }
    }
    return s0 + s1;
  }
  for (int at = threadIdx.x * 16; at < bytes; at += THREADS * 16) {
    if (at + 16 <= bytes) {
      float v[8];
      L::up(load16(p + at), v);
#pragma unroll
      for (int e = 0; e < L::N; e += 2) { s0 = fma((double)v[e], (double)v[e], s0); s1 = fma((double)v[e + 1], (double)v[e + 1], s1); }
    } else {
      for (int b = at; b < bytes; b += L::SIZE) { const double v = L::one(p + b); s0 = fma(v, v, s0); }
    }
  }
  return s0 + s1;
}

template <int DT, int THREADS>
__device__ __forceinline__ void piece_scale(const char *p, char *o, int bytes, float c) {
  typedef Lane<DT> L;
  constexpr int PER = PIECE / 16 / THREADS > 0 ? PIECE / 16 / THREADS : 1;
  if (bytes == PIECE) {
    Words x[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = load16(p + (i * THREADS + threadIdx.x) * 16);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float v[8];
      L::up(x[i], v);
#pragma unroll
      for (int e = 0; e < L::N; ++e) v[e] *= c;
      store16_past(o + (i * THREADS + threadIdx.x) * 16, L::down(v));
    }
    return;
  }
  for (int at = threadIdx.x * 16; at < bytes; at += THREADS * 16) {
    if (at + 16 <= bytes) {
      float v[8];
      L::up(load16(p + at), v);
#pragma unroll
      for (int e = 0; e < L::N; ++e) v[e] *= c;
      store16_past(o + at, L::down(v));
    } else {
      for (int b = at; b < bytes; b += L::SIZE) L::put(o + b, L::one(p + b) * c);
    }
  }
}

// The pieces [first, last) of the list, in order, from tensor `tensor`, its piece `piece` on: f(tensor, byte offset, bytes)
template <class F>
__device__ __forceinline__ void walk(const List &l, int group, F f) {
  const int64_t first = l.pieces * group / l.groups, last = l.pieces * (group + 1) / l.groups;
  int tensor = l.starts[group].tensor;
  int64_t piece = l.starts[group].piece;
  for (int64_t i = first; i < last; ++i) {
    Tensor t = l.tensors[tensor];
    while (piece * PIECE >= t.n * t.bytes) { t = l.tensors[++tensor]; piece = 0; }
    const int64_t at = piece * PIECE, rest = t.n * t.bytes - at;
    f(t, at, (int)(rest < PIECE ? rest : PIECE));
    ++piece;
  }
}

template <int THREADS>
__device__ __forceinline__ double group_sum(double s, double *shared) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = s;
  __syncthreads();
  double total = 0;
  for (int w = 0; w < THREADS / 64; ++w) total += shared[w];
  __syncthreads();
  return total;
}

template <int THREADS>
__device__ __forceinline__ double run_sum(const List &l, int group, double *shared) {
  double s = 0;
  walk(l, group, [&](const Tensor &t, int64_t at, int bytes) {
    if (t.dtype == CHM_F32) s += piece_sum<CHM_F32, THREADS>(t.in + at, bytes);
    else if (t.dtype == CHM_BF16) s += piece_sum<CHM_BF16, THREADS>(t.in + at, bytes);
    else s += piece_sum<CHM_F16, THREADS>(t.in + at, bytes);
  });
  return group_sum<THREADS>(s, shared);
}

// min(1, max_norm / (norm + 1e-6)), rounded once; not a number where the norm is none.  A norm beyond float32 of finite values still has one.
__device__ __forceinline__ float factor_of(double norm, float max_norm) {
  const double c = max_norm / (norm + 1e-6);
  return c > 1. ? 1.f : (float)c;
}

template <int THREADS>
__device__ __forceinline__ void run_scale(const List &l, int group, float c) {
  walk(l, group, [&](const Tensor &t, int64_t at, int bytes) {
    if (c == 1.f && t.out == t.in) return;
    if (t.dtype == CHM_F32) piece_scale<CHM_F32, THREADS>(t.in + at, t.out + at, bytes, c);
    else if (t.dtype == CHM_BF16) piece_scale<CHM_BF16, THREADS>(t.in + at, t.out + at, bytes, c);
    else piece_scale<CHM_F16, THREADS>(t.in + at, t.out + at, bytes, c);
  });
}

__global__ void __launch_bounds__(NT) k_sumsq(List l, double *sums) {
  __shared__ double shared[NT / 64];
  const double s = run_sum<NT>(l, blockIdx.x, shared);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__device__ __forceinline__ double all_sums(const double *sums, int n, double *shared) {
  double s = 0;
  for (int i = threadIdx.x; i < n; i += NT) s += sums[i];
  return group_sum<NT>(s, shared);
}

__global__ void __launch_bounds__(NT) k_total(const double *sums, int n, double *total) {
  __shared__ double shared[NT / 64];
  const double s = all_sums(sums, n, shared);
  if (threadIdx.x == 0) *total = s;
}

__global__ void __launch_bounds__(NT) k_scale(List l, const double *sums, int n, float max_norm, float *norm_out) {
  __shared__ double shared[NT / 64];
  const double norm = sqrt(all_sums(sums, n, shared));
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  // the pieces read last by the first pass come first: the cache still holds them
  run_scale<NT>(l, l.groups - 1 - blockIdx.x, factor_of(norm, max_norm));
}

// Whether every result shares memory with no tensor but its own, and with that one wholly or not at all
bool apart(const std::vector<Tensor> &tensors) {
  struct Span { uintptr_t from, to; bool out; };
  std::vector<Span> spans;
  for (const Tensor &t : tensors) {
    const uintptr_t in = (uintptr_t)t.in, out = (uintptr_t)t.out, bytes = (uintptr_t)(t.n * t.bytes);
    spans.push_back(Span{out, out + bytes, true});
    if (in != out) spans.push_back(Span{in, in + bytes, false});
  }
  std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.from < b.from; });
  uintptr_t end[2] = {0, 0};             // of the inputs and of the results so far
  for (const Span &s : spans) {
    if (s.from < end[1] || (s.out && s.from < end[0])) return false;
    if (s.to > end[s.out]) end[s.out] = s.to;
  }
  return true;
}

}  // namespace

struct chm_gradients {
  int device = 0;
  bool apart = true;                     // no result lies over another tensor: else clipping would read what it has written
  List list{};
  char *memory = nullptr;                // tensors, starts, sums
  double *sums = nullptr;
};

extern "C" int chm_load_gradients(const chm_gradient *in, int32_t count, chm_gradients **out) {
  if (!out) return CHM_ERR_ARG;
  *out = nullptr;
  if (count < 0 || (count > 0 && !in)) return CHM_ERR_ARG;
  try {
    std::vector<Tensor> tensors;
    std::vector<int64_t> first;          // piece at which each tensor starts
    int64_t pieces = 0;
    for (int i = 0; i < count; ++i) {
      const chm_gradient &t = in[i];
      if (t.dtype != CHM_F32 && t.dtype != CHM_BF16 && t.dtype != CHM_F16) return CHM_ERR_ARG;
      const int size = t.dtype == CHM_F32 ? 4 : 2;
      if (t.n < 0 || t.n > (INT64_MAX >> 4) || (t.n > 0 && !t.grad)) return CHM_ERR_ARG;
      if (((uintptr_t)t.grad | (uintptr_t)t.out) % size) return CHM_ERR_ARG;
      if (t.n == 0) continue;
      const int64_t p = (t.n * size + PIECE - 1) / PIECE;
      if (p > INT32_MAX) return CHM_ERR_ARG;
      tensors.push_back(Tensor{(const char *)t.grad, t.out ? (char *)t.out : (char *)t.grad, t.n, t.dtype, size});
      first.push_back(pieces);
      pieces += p;
    }
    chm_gradients *g = new chm_gradients;
    g->list.count = (int)tensors.size();
    g->list.pieces = pieces;
    g->list.groups = pieces < 1 ? 1 : pieces < GROUPS_MAX ? (int)pieces : GROUPS_MAX;
    std::vector<Start> starts(g->list.groups);
    size_t t = 0;
    for (int b = 0; b < g->list.groups; ++b) {
      const int64_t at = pieces * b / g->list.groups;
      while (t + 1 < tensors.size() && first[t + 1] <= at) ++t;
      starts[b] = Start{(int32_t)t, tensors.empty() ? 0 : (int32_t)(at - first[t])};
    }
    g->apart = apart(tensors);
    const size_t bt = tensors.size() * sizeof(Tensor), bs = starts.size() * sizeof(Start), bd = GROUPS_MAX * sizeof(double);
    std::vector<char> host(bt + bs);
    if (bt) memcpy(host.data(), tensors.data(), bt);
    memcpy(host.data() + bt, starts.data(), bs);
    if (hipGetDevice(&g->device) != hipSuccess || hipMalloc((void **)&g->memory, bd + bt + bs) != hipSuccess) {
      (void)hipGetLastError();
      delete g;
      return CHM_ERR_HIP;
    }
    if (hipMemcpy(g->memory + bd, host.data(), bt + bs, hipMemcpyHostToDevice) != hipSuccess) {
      (void)hipFree(g->memory);
      delete g;
      return CHM_ERR_HIP;
    }
    g->sums = (double *)g->memory;
    g->list.tensors = (const Tensor *)(g->memory + bd);
    g->list.starts = (const Start *)(g->memory + bd + bt);
    *out = g;
    return CHM_OK;
  } catch (const std::bad_alloc &) {
    return CHM_ERR_HIP;
  }
}

extern "C" int chm_gradient_sumsq(chm_gradients *g, double *d_sumsq, void *hip_stream) {
  if (!g || !d_sumsq) return CHM_ERR_ARG;
  hipStream_t st = (hipStream_t)hip_stream;
  hipLaunchKernelGGL(k_sumsq, dim3(g->list.groups), dim3(NT), 0, st, g->list, g->sums);
  hipLaunchKernelGGL(k_total, dim3(1), dim3(NT), 0, st, g->sums, g->list.groups, d_sumsq);
  return hipGetLastError() == hipSuccess ? CHM_OK : CHM_ERR_HIP;
}

extern "C" int chm_clip_gradients(chm_gradients *g, float max_norm, const double *d_sumsq, float *d_norm, void *hip_stream) {
  if (!g || !d_norm || !(max_norm >= 0) || !g->apart) return CHM_ERR_ARG;
  hipStream_t st = (hipStream_t)hip_stream;
  if (!d_sumsq) hipLaunchKernelGGL(k_sumsq, dim3(g->list.groups), dim3(NT), 0, st, g->list, g->sums);
  hipLaunchKernelGGL(k_scale, dim3(g->list.groups), dim3(NT), 0, st, g->list, d_sumsq ? d_sumsq : g->sums, d_sumsq ? 1 : g->list.groups,
                     max_norm, d_norm);
  return hipGetLastError() == hipSuccess ? CHM_OK : CHM_ERR_HIP;
}

extern "C" void chm_free_gradients(chm_gradients *g) {
  if (!g) return;
  (void)hipFree(g->memory);
  delete g;
}

// Rotary positions: pairs of a head's elements turned by the angle of their token.
//
//   theta = position * frequency;  a' = a cos - b sin,  b' = a sin + b cos
//
// Bytes are all there is to it (6 operations for 4 bytes and more), as long as the sine and cosine of a token and pair are worked out once, not once
// a head: a workgroup takes some tokens, works out their sines and cosines into shared memory (angles in float64, reduced to a turn, so
// that far positions keep their digits), and turns all heads of these tokens (or a share of them, where there are few tokens).
// 32,768 tokens of 40 heads of 128, three axes, bfloat16: 133 us, 671 MB read and written at 5.1 TB/s (a copy: 4.9); one token 4 us, start-up.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "chm_elements.h"
#include "chm_strided.h"

namespace {

using namespace chm_elements;

constexpr int PAIRS = 128, NT = 256;
constexpr int ANGLES = 1024;             // sines and cosines of a workgroup

struct Divide { uint32_t m; int32_t shift; };          // n / d for n below 2^31
Divide divide_by(uint32_t d) {
  if (d <= 1) return Divide{0, 0};
  int l = 0;
  while ((1ull << l) < d) ++l;
  return Divide{(uint32_t)((1ull << (31 + l)) / d + 1), l - 1};
}
__device__ __forceinline__ uint32_t over(Divide d, uint32_t n) { return d.m ? __umulhi(n, d.m) >> d.shift : n; }

struct RotaryCall {
  const char *x;
  char *out;
  const char *positions;
  int64_t x_token, x_head, out_token, out_head;        // bytes
  int64_t p_axis, p_token;                             // elements
  int64_t tokens;
  int32_t heads, head_dim, pairs, index_bits;
  int32_t tokens_each, heads_each, head_groups;        // of a workgroup; groups of heads
  int32_t turned, chunks;                              // pieces of a head that are turned, and all
  Divide by_pairs, by_chunks, by_heads;
  float sign;
  double turns[PAIRS];                                 // frequency / 2 pi
  uint8_t axis[PAIRS];
};

// up to N elements from p on, as float32; N of them without a branch
template <int DT> __device__ __forceinline__ void take(const char *p, int n, float *v) {
  typedef Lane<DT> L;
  if (n >= L::N) {
    L::up(load16(p), v);
  } else {
#pragma unroll
    for (int i = 0; i < L::N; ++i) v[i] = i < n ? L::one(p + i * L::SIZE) : 0.f;
  }
}
template <int DT> __device__ __forceinline__ void give(char *p, int n, const float *v) {
  typedef Lane<DT> L;
  if (n >= L::N) {
    store16(p, L::down(v));
  } else {
#pragma unroll
    for (int i = 0; i < L::N; ++i)
      if (i < n) L::put(p + i * L::SIZE, v[i]);
  }
}

template <int DT, int NEIGHBOURS>
__global__ void __launch_bounds__(NT) k_rotary(const RotaryCall c) {
  typedef Lane<DT> L;
  __shared__ float2 turn[ANGLES + 8];                  // (cosine, sine); a last piece reads behind the pairs
  const int64_t block = blockIdx.x / c.head_groups;
  const int group = blockIdx.x - (int)block * c.head_groups;
  const int64_t t0 = block * c.tokens_each;
  const int tokens = (int)(c.tokens - t0 < c.tokens_each ? c.tokens - t0 : c.tokens_each);
  for (int i = threadIdx.x; i < tokens * c.pairs; i += NT) {
    const int t = (int)over(c.by_pairs, i), pair = i - t * c.pairs;
    const int64_t at = c.axis[pair] * c.p_axis + (t0 + t) * c.p_token;
    const double pos = c.index_bits == 32 ? (double)((const int32_t *)c.positions)[at] : (double)((const int64_t *)c.positions)[at];
    const double turns = pos * c.turns[pair];
    float s, co;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
    turn[i] = float2{co, c.sign * s};
  }
  __syncthreads();
  const int h0 = group * c.heads_each, heads = c.heads - h0 < c.heads_each ? c.heads - h0 : c.heads_each;
  const int items = tokens * heads * c.chunks;
  for (int i = threadIdx.x; i < items; i += NT) {
    const int row = (int)over(c.by_chunks, i), piece = i - row * c.chunks;
    const int t = heads == c.heads_each ? (int)over(c.by_heads, row) : row / heads, h = row - t * heads;
    const char *x = c.x + (t0 + t) * c.x_token + (h0 + h) * c.x_head;
    char *out = c.out + (t0 + t) * c.out_token + (h0 + h) * c.out_head;
    float a[8], b[8];
    if (piece >= c.turned) {                           // behind the pairs
      const int d = 2 * c.pairs + (piece - c.turned) * L::N;
      take<DT>(x + (int64_t)d * L::SIZE, c.head_dim - d, a);
      give<DT>(out + (int64_t)d * L::SIZE, c.head_dim - d, a);
      continue;
    }
    if (NEIGHBOURS) {
      const int d = piece * L::N, n = 2 * c.pairs - d;
      const float2 *w = turn + t * c.pairs + d / 2;
      take<DT>(x + d * L::SIZE, n, a);
#pragma unroll
      for (int e = 0; e < L::N; e += 2) {
        const float2 u = w[e / 2];
        b[e] = a[e] * u.x - a[e + 1] * u.y;
        b[e + 1] = a[e] * u.y + a[e + 1] * u.x;
      }
      give<DT>(out + d * L::SIZE, n, b);
    } else {
      const int d = piece * L::N, n = c.pairs - d, second = (c.pairs + d) * L::SIZE;
      const float2 *w = turn + t * c.pairs + d;
      take<DT>(x + d * L::SIZE, n, a);
      take<DT>(x + second, n, b);
#pragma unroll
      for (int e = 0; e < L::N; ++e) {
        const float2 u = w[e];
        const float p = a[e], q = b[e];
        a[e] = p * u.x - q * u.y;
        b[e] = p * u.y + q * u.x;
      }
      give<DT>(out + d * L::SIZE, n, a);
      give<DT>(out + second, n, b);
    }
  }
}

template <int DT>
void launch(const RotaryCall &c, int neighbours, uint32_t groups, hipStream_t st) {
  if (neighbours) hipLaunchKernelGGL((k_rotary<DT, 1>), dim3(groups), dim3(NT), 0, st, c);
  else hipLaunchKernelGGL((k_rotary<DT, 0>), dim3(groups), dim3(NT), 0, st, c);
}

int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }

}  // namespace

extern "C" int chm_rotary_turn(const chm_rotary *r, int32_t backwards, void *hip_stream) {
  if (!r || (r->dtype != CHM_F32 && r->dtype != CHM_BF16 && r->dtype != CHM_F16) || (r->index_bits != 32 && r->index_bits != 64)) return CHM_ERR_ARG;
  if (r->pairing != CHM_PAIRS_HALVES && r->pairing != CHM_PAIRS_NEIGHBOURS) return CHM_ERR_ARG;
  if (r->tokens < 0 || r->tokens > INT32_MAX || r->heads < 0 || r->heads > INT32_MAX || r->axes < 1) return CHM_ERR_ARG;
  if (r->pairs < 1 || r->pairs > PAIRS || r->head_dim < 2 * r->pairs || r->head_dim > (1 << 20) || !r->frequencies) return CHM_ERR_ARG;
  const int size = r->dtype == CHM_F32 ? 4 : 2;
  if (((uintptr_t)r->x | (uintptr_t)r->out) % size || (uintptr_t)r->positions % (r->index_bits / 8)) return CHM_ERR_ARG;
  using chm_strided::countable;
  if (!countable(r->x_token, r->tokens) || !countable(r->x_head, r->heads) || !countable(r->out_token, r->tokens) || !countable(r->out_head, r->heads) ||
      !countable(r->positions_axis, r->axes) || !countable(r->positions_token, r->tokens)) return CHM_ERR_ARG;
  RotaryCall c{};
  for (int i = 0; i < r->pairs; ++i) {
    const int32_t a = r->axis ? r->axis[i] : 0;
    if (a < 0 || a >= r->axes || a > 255 || !isfinite(r->frequencies[i])) return CHM_ERR_ARG;
    c.turns[i] = r->frequencies[i] * 0.15915494309189533577;
    c.axis[i] = (uint8_t)a;
  }
  if (r->tokens == 0 || r->heads == 0) return CHM_OK;
  if (!r->x || !r->out || !r->positions) return CHM_ERR_ARG;
  const chm_strided::Dim none{1, 0}, tokens_in{r->tokens, r->x_token}, heads_in{r->heads, r->x_head}, tokens_out{r->tokens, r->out_token},
      heads_out{r->heads, r->out_head};
  const chm_strided::Tensor in(r->x, r->head_dim, size, {tokens_in, heads_in, none}), out(r->out, r->head_dim, size, {tokens_out, heads_out, none}),
      positions(r->positions, 1, r->index_bits / 8, {chm_strided::Dim{r->axes, r->positions_axis}, chm_strided::Dim{r->tokens, r->positions_token}, none});
  if (!out.apart() || chm_strided::share(out, positions)) return CHM_ERR_ARG;
  // in place: every element is read by whoever stores it
  const bool same = r->x == r->out && (r->tokens == 1 || r->x_token == r->out_token) && (r->heads == 1 || r->x_head == r->out_head);
  if (!same && chm_strided::share(out, in)) return CHM_ERR_ARG;

  const int n = 16 / size;
  c.x = (const char *)r->x;
  c.out = (char *)r->out;
  c.positions = (const char *)r->positions;
  const auto step = [](int64_t stride, int64_t n) { return n < 2 ? 0 : stride; };
  c.x_token = step(r->x_token, r->tokens) * size; c.x_head = step(r->x_head, r->heads) * size;
  c.out_token = step(r->out_token, r->tokens) * size; c.out_head = step(r->out_head, r->heads) * size;
  c.p_axis = step(r->positions_axis, r->axes); c.p_token = step(r->positions_token, r->tokens);
  c.tokens = r->tokens;
  c.heads = (int32_t)r->heads; c.head_dim = r->head_dim; c.pairs = r->pairs; c.index_bits = r->index_bits;
  c.turned = (int32_t)(r->pairing == CHM_PAIRS_NEIGHBOURS ? up(2 * r->pairs, n) : up(r->pairs, n));
  c.chunks = c.turned + (int32_t)(same ? 0 : up(r->head_dim - 2 * r->pairs, n));
  // Some 1,024 pieces a workgroup (4 a thread) and at least as many angles' worth of tokens as there are threads; fewer heads a workgroup
  // while there are fewer workgroups than compute units
  const int64_t per_token = (int64_t)c.heads * c.chunks;
  int64_t each = up(1024, per_token);
  if (each > ANGLES / r->pairs) each = ANGLES / r->pairs;
  if (each > r->tokens) each = r->tokens;
  c.tokens_each = (int32_t)each;
  const int64_t blocks = up(r->tokens, each);
  int64_t heads_each = up(r->heads, 1);
  const int64_t least = up(NT, each * c.chunks);       // heads that give every thread a piece
  while (heads_each > least && blocks * up(r->heads, heads_each) < 256) heads_each = up(heads_each, 2);
  const int64_t most = (1 << 22) / (each * c.chunks);  // pieces of a workgroup are counted in 31 bits
  if (heads_each > most) heads_each = most < 1 ? 1 : most;
  c.heads_each = (int32_t)heads_each;
  c.head_groups = (int32_t)up(r->heads, heads_each);
  const int64_t groups = blocks * c.head_groups;
  if (groups * NT > UINT32_MAX) return CHM_ERR_ARG;
  c.by_pairs = divide_by(c.pairs);
  c.by_chunks = divide_by(c.chunks);
  c.by_heads = divide_by((uint32_t)heads_each);
  c.sign = backwards ? -1.f : 1.f;
  hipStream_t st = (hipStream_t)hip_stream;
  const int neighbours = r->pairing == CHM_PAIRS_NEIGHBOURS;
  if (r->dtype == CHM_F32) launch<CHM_F32>(c, neighbours, (uint32_t)groups, st);
  else if (r->dtype == CHM_BF16) launch<CHM_BF16>(c, neighbours, (uint32_t)groups, st);
  else launch<CHM_F16>(c, neighbours, (uint32_t)groups, st);
  return hipGetLastError() == hipSuccess ? CHM_OK : CHM_ERR_HIP;
}

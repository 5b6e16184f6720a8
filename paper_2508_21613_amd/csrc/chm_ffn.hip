// Gated feed-forward block: what its passes consist of, the kernels for few tokens, the packing of unaligned operands, the entry points.
//
//   forward    h = act(x Wg^T) * (x Wu^T)      one product with two weights, activation and product in its epilogue
//              y = h Wd^T
//   backward   dh = dy Wd, and in its epilogue  h = act(g) u,  du = dh act(g),  dg = dh u act'(g)
//              dx = [dg du] [Wg; Wu]            one product over 2 F sums
//              [dWg; dWu] = [dg du]^T x         one product with 2 F rows
//              dWd = dy^T h
// All of them are bound by the matrix cores for a micro-batch of tokens (chm_gemm.h) and by reading the weights for a few.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/chm_measure.h"
#include "chm_elements.h"
#include "chm_gemm.h"
#include "chm_overlap.h"

namespace {

using namespace chm_elements;
using chm_gemm::f4;
using chm_gemm::s8;

// ---------------------------------------------------------------------------------------------- few tokens
// A wavefront takes 16 features (rows of a weight; fewer with few tokens) and a share of the sums, and reads its part of the weight straight into
// the first operand of the matrix instructions: every byte of a weight is read once, by one wavefront, 64 contiguous bytes a
// lane quad and step.  The tokens (16 for each instruction, absent ones are zero and not loaded) come from the cache.  The
// wavefronts of a workgroup share the sums and add them up through shared memory, in order.  Weights may start anywhere.
// Tokens up to which these kernels run rather than the tiles: 8, 24 with small weights, 48 with smaller ones.  From there on the tokens'
// fragments, which every wavefront reads for itself, cost more than the tiles' fixed time (us, these kernels and tiles: 512 x 1,376, 48 tokens
// 15 and 15, 64 tokens 18 and 15; 1,024 x 2,752, 24 tokens 19 and 19, 32 tokens 21 and 19; 2,048 x 5,504, 8 tokens 23 and 28, 10 tokens 28 and
// 28, 16 tokens 31 and 26; 4,096 x 11,008, 8 tokens 62 and 67, 16 tokens 66 and 66, 20 tokens 79 and 68; 8,192 x 22,016, 5 tokens 213 and 224, 8 tokens
// 233 and 224).  32 with large weights that the tiles would have to pack first (4,001 x 11,001, 32 tokens 168 and 184, 40 tokens 212 and 186).
bool few_tokens(int64_t tokens, int64_t width, int64_t features, bool packs) {
  const int64_t weight = width * features;
  return tokens <= (weight <= 1 << 20 ? 48 : weight <= 1 << 23 ? 24 : packs && weight > 1 << 25 ? 32 : 8);
}

int64_t up8(int64_t n) { return (n + 7) & ~7ll; }

struct FewCall {
  const uint16_t *x, *w0, *w1;
  int64_t ldx, ld0, ld1;
  uint16_t *out;
  Kept kept;
  int64_t ldo;
  int32_t tokens, rows, k, act;
};

// 8 elements at k of a row of `n`, zeros beyond
__device__ __forceinline__ s8 take8(const uint16_t *row, int k, int n) {
  if (k + 8 <= n) return __builtin_bit_cast(s8, load16((const char *)(row + k)));
  s8 v = {};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (k + e < n) v[e] = (short)((const CHM_GLOBAL uint16_t *)row)[k + e];
  return v;
}

__device__ __forceinline__ float act(int kind, float g) {
  if (kind == CHM_ACT_SILU) return chm_gemm::act_of<CHM_ACT_SILU>(g);
  return kind == CHM_ACT_GELU ? chm_gemm::act_of<CHM_ACT_GELU>(g) : chm_gemm::act_of<CHM_ACT_GELU_TANH>(g);
}

__device__ __forceinline__ void keep_pair(const FewCall &c, int64_t m, int64_t f, float g, float u) {
  const uint32_t bg = chm_gemm::upper24(g), bu = chm_gemm::upper24(u);
  char *p = chm_gemm::kept_at(c.kept, m, f);
  const int e = (int)f & 7;
  ((uint16_t *)p)[e] = (uint16_t)(bg >> 16);
  ((uint16_t *)(p + 1024))[e] = (uint16_t)(bu >> 16);
  ((uint8_t *)(p + 2048))[e] = (uint8_t)(bg >> 8);
  ((uint8_t *)(p + 2048))[8 + e] = (uint8_t)(bu >> 8);
}

// wavefronts of a workgroup at most: two steps and more of several tiles take more registers than 16 of them leave
constexpr int few_waves_most(int tiles) { return tiles == 1 ? 16 : 8; }

// 64 sums of each slice: 16 of every lane's feature and of its token of each tile.  Eight that would end behind the row are its last eight
// instead; what of these belongs to an earlier lane or step is set to zero before the product, which heeds no order of the sums.
template <int TWO, int TILES, int SLICES, int ENDS>
struct FewStep {
  s8 a[TWO + 1][2], b[TILES][2];
  template <bool SHORT> __device__ __forceinline__ void load(const FewCall &c, const uint16_t *w0, const uint16_t *w1, int k, int q, int r) {
    int at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      at[h] = first(k, h, q, r);
      if (ENDS && !SHORT) at[h] = at[h] < c.k - 8 ? at[h] : c.k - 8;
      a[0][h] = take<SHORT>(w0, at[h], c.k);
      if (TWO) a[TWO][h] = take<SHORT>(w1, at[h], c.k);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int token = t * 16 + r % (16 / SLICES), there = token < c.tokens ? token : c.tokens - 1;     // an absent one: the last again, its sums are dropped
      const uint16_t *x = c.x + there * c.ldx;
#pragma unroll
      for (int h = 0; h < 2; ++h) b[t][h] = take<SHORT>(x, at[h], c.k);
    }
  }
  template <class T> __device__ __forceinline__ void multiply(f4 (&acc)[2][TILES]) const {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w <= TWO; ++w) acc[w][t] = T::mfma(a[w][h], b[t][h], acc[w][t]);
  }
  // the step that starts at sum k
  template <class T> __device__ __forceinline__ void multiply(f4 (&acc)[2][TILES], const FewCall &c, int k, int q, int r) {
    if (ENDS && k + 64 * SLICES > c.k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int drop = first(k, h, q, r) - (c.k - 8);
        uint4 keep;
        keep.x = (drop > 0 ? 0 : 0xffffu) | (drop > 1 ? 0 : 0xffff0000u);
        keep.y = (drop > 2 ? 0 : 0xffffu) | (drop > 3 ? 0 : 0xffff0000u);
        keep.z = (drop > 4 ? 0 : 0xffffu) | (drop > 5 ? 0 : 0xffff0000u);
        keep.w = (drop > 6 ? 0 : 0xffffu) | (drop > 7 ? 0 : 0xffff0000u);
        const s8 mask = __builtin_bit_cast(s8, keep);
#pragma unroll
        for (int w = 0; w <= TWO; ++w) a[w][h] &= mask;
#pragma unroll
        for (int t = 0; t < TILES; ++t) b[t][h] &= mask;
      }
    }
    multiply<T>(acc);
  }
  static __device__ __forceinline__ int first(int k, int h, int q, int r) { return k + r / (16 / SLICES) * 64 + h * 32 + q * 8; }
  template <bool SHORT> static __device__ __forceinline__ s8 take(const uint16_t *row, int at, int n) {
    return SHORT ? take8(row, at, n) : __builtin_bit_cast(s8, load16((const char *)(row + at)));
  }
};

template <class T, int TWO, int TILES, int SLICES, int ENDS>
__global__ void __launch_bounds__(64 * few_waves_most(TILES)) k_few_tokens(FewCall c) {
  extern __shared__ float part[];             // [wavefronts][TWO + 1][TILES][64][4]
  // uniform: a matrix instruction does not heed which lanes are switched off
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int q = lane >> 4, r = lane & 15;
  constexpr int EACH = 16 / SLICES;           // features, and tokens of a tile
  const int f0 = blockIdx.x * EACH, f = f0 + r % EACH < c.rows ? f0 + r % EACH : c.rows - 1;
  const uint16_t *w0 = c.w0 + f * c.ld0, *w1 = TWO ? c.w1 + f * c.ld1 : nullptr;
  f4 acc[2][TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) acc[0][t] = acc[1][t] = f4{0.f, 0.f, 0.f, 0.f};

  // DEPTH steps of 64 sums a slice are under way.  All loads are issued whatever the number of steps (a step too many reads the last one
  // again), and none depends on a branch: else the waits in front of the matrix instructions would be for all of them.  Workgroups
  // begin at different sums, so that they do not all ask the same channels of the cache for the tokens.
  constexpr int DEPTH = TWO && TILES > 2 ? 3 : 4;
  const int steps = (c.k + 64 * SLICES - 1) / (64 * SLICES);
  if (ENDS && c.k < 8) {
    if (wave == 0) {
      FewStep<TWO, TILES, SLICES, ENDS> only;
      only.template load<true>(c, w0, w1, 0, q, r);
      only.template multiply<T>(acc);
    }
  } else if (wave < steps) {
    const int turn = (int)((blockIdx.x >> 3) % (uint32_t)steps);
    const auto at = [&](int i) {
      i = (i < steps ? i : steps - 1) + turn;
      return (i < steps ? i : i - steps) * 64 * SLICES;
    };
    FewStep<TWO, TILES, SLICES, ENDS> set[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) set[d].template load<false>(c, w0, w1, at(wave + d * waves), q, r);
    int i = wave;
    for (; i + DEPTH * waves < steps; i += DEPTH * waves)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        set[d].template multiply<T>(acc, c, at(i + d * waves), q, r);
        set[d].template load<false>(c, w0, w1, at(i + (d + DEPTH) * waves), q, r);
      }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (i + d * waves < steps) set[d].template multiply<T>(acc, c, at(i + d * waves), q, r);
  }

#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int w = 0; w <= TWO; ++w) *(f4 *)(part + ((((wave * (TWO + 1) + w) * TILES) + t) * 64 + lane) * 4) = acc[w][t];
  __syncthreads();
  // one value (pair) a thread: feature o % EACH, token o / EACH
  for (int o = threadIdx.x; o < EACH * EACH * TILES; o += blockDim.x) {
    const int feature = o % EACH, token = o / EACH;
    if (token >= c.tokens) continue;
    if (f0 + feature >= c.rows) {             // kept projections have rows of whole words of 8, zeros behind
      if (TWO && c.kept.p && f0 + feature < ((c.rows + 7) & ~7)) keep_pair(c, token, f0 + feature, 0.f, 0.f);
      continue;
    }
    const int at = ((token >> 4) * 64 + (feature >> 2) * 16 + (token & 15)) * 4 + (feature & 3);
    float s0 = 0.f, s1 = 0.f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
      for (int s = 0; s < SLICES; ++s) {      // EACH features and tokens on: EACH lanes for the tokens, EACH / 4 times 16 for the features
        const float *p = part + w * (TWO + 1) * TILES * 256 + at + s * (EACH + EACH / 4 * 16) * 4;
        s0 += p[0];
        if (TWO) s1 += p[TILES * 256];
      }
    const int64_t col = f0 + feature;
    if (TWO) {
      c.out[token * c.ldo + col] = T::down(act(c.act, s0) * s1);
      if (c.kept.p) keep_pair(c, token, col, s0, s1);
    } else {
      c.out[token * c.ldo + col] = T::down(s0);
    }
  }
}

// wavefronts of a workgroup: some 16 a compute unit over all, with four steps of 64 sums each at least
int few_waves(int64_t groups, int64_t steps, int tiles) {
  int w = 1;
  while (w < few_waves_most(tiles) && groups * w < 4096 && steps >= w * 8) w <<= 1;
  return w;
}

// Up to 8 tokens the 16 rows of the operands may be 8 or 4 features (and as many tokens) of 2 or 4 slices of the sums; of the products of all
// pairs of slices, those of a slice with itself are added up.  That gives 2 or 4 times the workgroups and longer runs of a weight's row, but each
// of them loads 2 or 4 times as many tokens.  The least of: how unevenly the workgroups fall on 256 compute units, times what short runs
// cost (more where rows do not start on whole lines of 128 bytes), times what the tokens cost.
// Measured (us; one slice, two, four in both launches): 1 token, 2,048 x 5,504 24.3, 19.0, 19.4; 1,024 x 2,752 12.4, 10.4, 9.6; 1,000 x 2,731
// 18.8, 13.4, 10.3; 3,000 x 8,000 38.8, 33.6, 32.2; 4,096 x 11,008 55.8, 55.5, 54.4; 8,192 x 22,016 212, 202, 189.  4 tokens, the same widths:
// 25.7, 19.4, 21.8; 13.4, 11.3, 10.5; 19.5, 14.2, 10.8; 41.5, 37.8, 40.3; 57.0, 59.8, 65.7; 217, 217, 233.  8 tokens, two last widths: 60.5, 67.8; 227, 248.
int few_slices(int two, const FewCall &c) {
  const bool lines = (c.ld0 % 64 == 0) && (c.ld1 % 64 == 0);
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= 4 && s * c.tokens <= 16; s <<= 1) {
    const double groups = (double)((c.rows * (int64_t)s + 15) / 16), loaded = c.tokens * s;
    const double cost = ceil(groups / 256) / groups * (1 + (lines ? 0.1 : 0.5) / s) * (1 + (two ? 0.001 : 0.002) * loaded * loaded);
    if (cost < least) least = cost, best = s;
  }
  return best;
}

template <class T, int TWO, int TILES, int SLICES>
void launch_few(const FewCall &c, hipStream_t st) {
  const int64_t each = 16 / SLICES, groups = (up8(c.rows) + each - 1) / each;          // kept projections have zeros up to a whole word
  const int w = few_waves(groups, (c.k + 64 * SLICES - 1) / (64 * SLICES), TILES);
  const size_t bytes = (size_t)w * (TWO + 1) * TILES * 1024;
  if (c.k % (64 * SLICES)) hipLaunchKernelGGL((k_few_tokens<T, TWO, TILES, SLICES, 1>), dim3((uint32_t)groups), dim3(w * 64), bytes, st, c);
  else hipLaunchKernelGGL((k_few_tokens<T, TWO, TILES, SLICES, 0>), dim3((uint32_t)groups), dim3(w * 64), bytes, st, c);
}
int few_blocks(const FewCall &c) { return (c.tokens + 15) / 16; }
template <class T, int TWO>
bool launch_few(const FewCall &c, hipStream_t st) {
  const int tiles = few_blocks(c), slices = few_slices(TWO, c);
  if (slices == 4) launch_few<T, TWO, 1, 4>(c, st);
  else if (slices == 2) launch_few<T, TWO, 1, 2>(c, st);
  else if (tiles == 1) launch_few<T, TWO, 1, 1>(c, st);
  else if (tiles == 2) launch_few<T, TWO, 2, 1>(c, st);
  else launch_few<T, TWO, 3, 1>(c, st);
  return hipGetLastError() == hipSuccess;
}

// ---------------------------------------------------------------------------------------------- packing
// An operand whose rows do not start on 16 bytes or are no whole words of 8 elements is copied into rows that are, with zeros
// behind: the copy costs its bytes twice, a product reads them some dozens of times.
struct PackCall {
  struct { const uint16_t *in; uint16_t *out; int64_t ld, rows; int32_t cols, words, groups; } m[5];
  int32_t count;
};
constexpr int PACK_WORDS = 4 * 256;           // 16-byte words of a workgroup

// all operands of a pass in one launch, one behind the other
__global__ void __launch_bounds__(256) k_pack(PackCall c) {
  int g = blockIdx.x, i = 0;
  while (i + 1 < c.count && g >= c.m[i].groups) g -= c.m[i++].groups;
  const int words = c.m[i].words, cols = c.m[i].cols;
  const int64_t all = c.m[i].rows * words, first = (int64_t)g * PACK_WORDS + threadIdx.x;
  s8 v[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int64_t w = first + u * 256;
    if (w < all) v[u] = take8(c.m[i].in + w / words * c.m[i].ld, (int)(w % words) * 8, cols);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int64_t w = first + u * 256;
    if (w < all) *(s8 *)(c.m[i].out + w * 8) = v[u];
  }
}

// ---------------------------------------------------------------------------------------------- sums split over workgroups
template <class T>
__global__ void __launch_bounds__(256) k_join_parts(const float *part, int splits, int64_t rows, int64_t ld_part, int cols, uint16_t *out,
                                                    int64_t ld_out) {
  const int words = (int)(ld_part / 8);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * words; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / words;
    const int col = (int)(i - row * words) * 8;
    const float *p = part + row * ld_part + col;
    f4 a = *(const f4 *)p, b = *(const f4 *)(p + 4);
    for (int s = 1; s < splits; ++s) {
      p += rows * ld_part;
      a += *(const f4 *)p;
      b += *(const f4 *)(p + 4);
    }
    const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    uint16_t *o = out + row * ld_out + col;
    if (col + 8 <= cols) {
      store16((char *)o, __builtin_bit_cast(Words, chm_gemm::pack8<T>(v)));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < cols) o[e] = T::down(v[e]);
    }
  }
}

uint32_t copy_groups(int64_t words) {
  const int64_t g = (words + 255) / 256;
  return (uint32_t)(g < 1 ? 1 : g < 8192 ? g : 8192);
}

// ---------------------------------------------------------------------------------------------- passes

struct Matrix { const void *p; int64_t ld, rows, cols; };

bool needs_pack(const Matrix &m) { return (uintptr_t)m.p % 16 || m.ld % 8 || m.cols % 8 || m.ld > GEMM_LD_MAX; }

// whether the forward pass runs on the kernels for few tokens
bool takes_few(const chm_ffn *f) {
  const int64_t D = f->width, F = f->features;
  const bool packs = needs_pack({f->w_gate, f->ld_gate, F, D}) || needs_pack({f->w_up, f->ld_up, F, D}) || needs_pack({f->w_down, f->ld_down, D, F});
  return few_tokens(f->tokens, D, F, packs);
}

// Hands out scratch, in a fixed order; with no base it only counts
struct Arena {
  char *base;
  uint64_t used = 0;
  void *take(uint64_t bytes) {
    void *p = base ? base + used : nullptr;
    used += (bytes + 255) & ~255ull;
    return p;
  }
};

int64_t kept_blocks(const chm_ffn *f) { return (f->features + 31) / 32; }
uint64_t kept_bytes(const chm_ffn *f) { return (uint64_t)((f->tokens + 15) / 16) * kept_blocks(f) * 3072; }
Kept kept_of(const chm_ffn *f) { return Kept{(char *)f->saved, kept_blocks(f)}; }

struct Pass {
  const chm_ffn *f;
  Arena arena;
  hipStream_t st;
  bool run, ok = true;
  bool fits = true;                        // every launch's threads can be counted in 32 bits, as a grid's are; else the calls refuse

  chm_ffn_kernels chosen{0, {0, 0}, {0, 0}, {-1, -1, -1, -1}, {0, 0, 0, 0}};

  Pass(const chm_ffn *f_, char *base, hipStream_t st_, bool run_) : f(f_), arena{base}, st(st_), run(run_) {}

  // the matrix itself, or a packed copy of it: made by the next flush().  Without tokens no operand is read, and none need be there.
  PackCall pack{};
  Matrix packed(const Matrix &m, bool must = false) {
    if (f->tokens == 0 || (!must && !needs_pack(m))) return m;
    Matrix o{nullptr, up8(m.cols), m.rows, up8(m.cols)};
    o.p = arena.take((uint64_t)o.rows * o.ld * 2);
    const int64_t words = o.rows * (o.ld / 8);
    if (words) {
      auto &p = pack.m[pack.count++];
      p.in = (const uint16_t *)m.p;
      p.out = (uint16_t *)o.p;
      p.ld = m.ld;
      p.rows = m.rows;
      p.cols = (int32_t)m.cols;
      p.words = (int32_t)(o.ld / 8);
      p.groups = (int32_t)((words + PACK_WORDS - 1) / PACK_WORDS);
    }
    return o;
  }
  void flush() {
    if (!run || !pack.count) return;
    uint32_t groups = 0;
    for (int i = 0; i < pack.count; ++i) groups += pack.m[i].groups;
    hipLaunchKernelGGL(k_pack, dim3(groups), dim3(256), 0, st, pack);
    ok = ok && hipGetLastError() == hipSuccess;
  }
  // two weights of one product: rows of equal length in memory, so both are packed where one has to be
  void packed_pair(Matrix &a, Matrix &b) {
    const bool must = a.ld != b.ld || needs_pack(a) || needs_pack(b);
    a = packed(a, must);
    b = packed(b, must);
  }

  // How a launch's products are laid out: kind of tile, parts of the first one's sums, and the time that takes.
  struct Layout { int tile = TILE_256, splits = 1; double us = 1e30; };

  // A tile takes a time for every step of 64 sums and one for its start and end, and 256 of them are worked on at a time, or 512 (two a compute
  // unit): 256 x 256 1.3 us a step and 10, 128 x 128 1.03 and 4.6, or alone on its compute unit, with more steps under way, 0.58 and 4,
  // 64 x 64 0.6 and 4 (4 and 1 more for dh, whose tiles read and write most at their end).
  // Measured against that (us): 1,024 x 22,016 x 4,096 186 and 211 expected, 176 and 197 taken; 512 x 22,016 93 and 113, 86 and 99; 256 x
  // 22,016 93 and 71, 81 and 61; 1,024 x 4,096 x 4,096 93, 42 and 41 (alone), 76, 44 and 40; 4,096 x 11,008 x 512 61 and 72, 67 and 72.
  // Sums are split (a first product with a plain 16-bit output only) 512 a part at least; the parts are written and read once more.
  // Whole steps against every choice of tile and split for dx and the weight gradients, with dx in a launch of its own and without: at 256 to
  // 2,048 tokens and widths of 1,000 to 4,096 this one is within 2% of the best (8% at 256 x 4,096 x 11,008), which is never the one apart.
  Layout layout(int products, const GemmCall *call, int count, bool may_split) const {
    static const double STEP[4] = {1.3, 1.03, 0.58, 0.6}, ENDS[4] = {10, 4.6, 4, 4};
    Layout best;
    for (int tile = TILE_256; tile <= TILE_64; ++tile) {
      if (tile == TILE_64 && products == GEMM_BACK) break;
      const int bits = side_bits(tile), at_once = tile == TILE_128 || tile == TILE_64 ? 512 : 256;
      const double ends = ENDS[tile] + (products != GEMM_DH || tile == TILE_256 ? 0 : tile == TILE_64 ? 1 : 4);
      const int64_t most = (1 << bits) - 1;
      for (int s = 1; s <= 8; ++s) {
        if (s > 1 && (!may_split || sums(call[0]) < 512 * (int64_t)s)) break;
        double work = 0, longest = 0, us;
        int64_t tiles = 0, groups = 0;
        for (int i = 0; i < count; ++i) {
          const int parts = i == 0 ? s : 1;
          const int64_t n = products == GEMM_GATE_UP ? 2 * call[i].n : call[i].n;
          const int64_t t = ((call[i].m + most) >> bits) * ((n + most) >> bits) * parts;
          groups += ((t / parts + 7) & ~7ll) * parts;
          const double unit = (double)((sums(call[i]) + 63) / 64 + parts - 1) / parts * STEP[tile] + ends;
          work += t * unit;
          tiles += t;
          if (t && unit > longest) longest = unit;
        }
        if (groups * (tile == TILE_64 ? 256 : 512) > UINT32_MAX) continue;
        if (tile == TILE_64) {             // the third of a compute unit begins where the first ends
          us = tiles <= 256 ? 0.8 * longest : tiles <= 512 ? longest : tiles * longest / 512;
        } else if (count == 1) {           // equal tiles: whole rounds, one of single tiles where two fit goes faster
          const int64_t rest = tiles % at_once;
          us = tiles / at_once * longest + (rest == 0 ? 0 : tile == TILE_128 && rest <= 256 ? 0.7 * longest : longest);
        } else {
          us = work / at_once > longest ? work / at_once : longest;
        }
        if (s > 1) us += 3 + (double)s * call[0].m * up8(call[0].n) * 8 / 4.5e6;
        if (us < best.us) best = Layout{tile, s, us};
      }
    }
    return best;
  }

  static int side_bits(int tile) { return tile == TILE_256 ? 8 : tile == TILE_64 ? 6 : 7; }

  void launch(int products, GemmGroup &g) {
    const Layout l = layout(products, g.call, g.count, products == GEMM_OUT || products == GEMM_BACK);
    fits = fits && l.us < 1e30;
    if (!fits) return;
    chosen.tile[products] = l.tile;
    chosen.splits[products] = l.splits;
    const int side = 1 << side_bits(l.tile);
    g.first[0] = 0;
    for (int i = 0; i < g.count; ++i) {
      GemmCall &c = g.call[i];
      const int64_t n = products == GEMM_GATE_UP ? 2 * c.n : c.n;
      c.tiles_m = (int32_t)((c.m + side - 1) / side);
      c.tiles_n = (int32_t)((n + side - 1) / side);
      c.splits = i == 0 ? l.splits : 1;
      c.act = f->activation;
      if (c.splits > 1) {
        c.ld_part = up8(c.n);
        c.part = (float *)arena.take((uint64_t)c.splits * c.m * c.ld_part * 4);
      }
      g.first[i + 1] = g.first[i] + ((c.tiles_m * c.tiles_n + 7) & ~7) * c.splits;
    }
    if (!run || g.first[g.count] == 0) return;
    ok = ok && (f->dtype == CHM_BF16 ? gemm_launch_bf16 : gemm_launch_f16)(products, l.tile, g, st);
    const GemmCall &c = g.call[0];
    if (c.splits > 1) {
      const dim3 grid(copy_groups(c.m * (c.ld_part / 8)));
      if (f->dtype == CHM_BF16)
        hipLaunchKernelGGL((k_join_parts<chm_gemm::Bf16>), grid, dim3(256), 0, st, c.part, c.splits, c.m, c.ld_part, (int)c.n_real, (uint16_t *)c.c[0], c.ldc);
      else
        hipLaunchKernelGGL((k_join_parts<chm_gemm::F16>), grid, dim3(256), 0, st, c.part, c.splits, c.m, c.ld_part, (int)c.n_real, (uint16_t *)c.c[0], c.ldc);
      ok = ok && hipGetLastError() == hipSuccess;
    }
  }
  static int64_t sums(const GemmCall &c) { return (c.a.k > c.b.k ? c.a.k : c.b.k) * c.runs; }

  void forward(void *y, int64_t ld_y) {
    const int64_t T = f->tokens, D = f->width, F = f->features, F8 = up8(F);
    const Kept kept = kept_of(f);
    uint16_t *h = (uint16_t *)arena.take((uint64_t)T * F8 * 2);
    if (takes_few(f)) {
      if (T == 0) return;
      FewCall c{};
      c.tokens = (int32_t)T;
      c.act = f->activation;
      c.x = (const uint16_t *)f->x; c.ldx = f->ld_x;
      c.w0 = (const uint16_t *)f->w_gate; c.ld0 = f->ld_gate;
      c.w1 = (const uint16_t *)f->w_up; c.ld1 = f->ld_up;
      c.out = h; c.ldo = F8;
      c.kept = kept;
      c.rows = (int32_t)F; c.k = (int32_t)D;
      few(0, c);
      if (run) ok = f->dtype == CHM_BF16 ? launch_few<chm_gemm::Bf16, 1>(c, st) : launch_few<chm_gemm::F16, 1>(c, st);
      FewCall d{};
      d.tokens = (int32_t)T;
      d.x = h; d.ldx = F8;
      d.w0 = (const uint16_t *)f->w_down; d.ld0 = f->ld_down;
      d.out = (uint16_t *)y; d.ldo = ld_y;
      d.rows = (int32_t)D; d.k = (int32_t)F;
      few(1, d);
      if (run) ok = ok && (f->dtype == CHM_BF16 ? launch_few<chm_gemm::Bf16, 0>(d, st) : launch_few<chm_gemm::F16, 0>(d, st));
      return;
    }
    const Matrix x = packed({f->x, f->ld_x, T, D}), wd = packed({f->w_down, f->ld_down, D, F});
    Matrix wg{f->w_gate, f->ld_gate, F, D}, wu{f->w_up, f->ld_up, F, D};
    packed_pair(wg, wu);
    flush();
    GemmGroup first{}, second{};
    first.count = second.count = 1;
    GemmCall &c = first.call[0], &d = second.call[0];
    c.a = GemmOperand{{x.p, x.p}, x.ld, x.cols};
    c.b = GemmOperand{{wg.p, wu.p}, wg.ld, wg.cols};
    c.m = T; c.n = F;
    c.runs = 1;
    c.h = h; c.kept = kept; c.ldi = F8;
    launch(GEMM_GATE_UP, first);
    d.a = GemmOperand{{h, h}, F8, F8};
    d.b = GemmOperand{{wd.p, wd.p}, wd.ld, wd.cols};
    d.m = T; d.n = D;
    d.runs = 1;
    out(d, y, ld_y, D);
    launch(GEMM_OUT, second);
  }

  void few(int which, const FewCall &c) {
    chosen.few = few_blocks(c);
    chosen.few_slices[which] = few_slices(!which, c);
    chosen.few_ends[which] = c.k % (64 * chosen.few_slices[which]) != 0;
  }

  // one 16-bit output of `cols` columns
  void out(GemmCall &c, void *p, int64_t ld, int64_t cols) {
    c.c[0] = c.c[1] = p;
    c.ldc = ld;
    c.m_first = c.m_real = c.m;
    c.n_real = cols;
  }

  void backward(const chm_ffn_gradients *g) {
    const int64_t T = f->tokens, D = f->width, F = f->features, F8 = up8(F);
    const Kept kept = kept_of(f);
    uint16_t *h = (uint16_t *)arena.take((uint64_t)T * F8 * 2), *d = (uint16_t *)arena.take((uint64_t)T * F8 * 4);
    const Matrix x = packed({f->x, f->ld_x, T, D}), dy = packed({g->dy, g->ld_dy, T, D}), wd = packed({f->w_down, f->ld_down, D, F});
    Matrix wg{f->w_gate, f->ld_gate, F, D}, wu{f->w_up, f->ld_up, F, D};
    packed_pair(wg, wu);
    flush();

    GemmGroup first{}, second{};
    first.count = 1;
    second.count = 3;
    GemmCall &a = first.call[0];           // dh, and h, dg, du
    a.a = GemmOperand{{dy.p, dy.p}, dy.ld, dy.cols};
    a.b = GemmOperand{{wd.p, wd.p}, wd.ld, D};
    a.m = T; a.n = F8; a.n_real = F;
    a.runs = 1;
    a.h = h; a.kept = kept; a.ldi = F8;
    a.dgate = d; a.dup = d + F8; a.ldd = 2 * F8;
    launch(GEMM_DH, first);

    GemmCall &i = second.call[0];          // dx
    i.a = GemmOperand{{d, d + F8}, 2 * F8, F8};
    i.b = GemmOperand{{wg.p, wu.p}, wg.ld, F};
    i.m = T; i.n = wg.cols;
    i.runs = 2;
    out(i, g->dx, g->ld_dx, D);

    GemmCall &b = second.call[1];          // dWd
    b.a = GemmOperand{{dy.p, dy.p}, dy.ld, T};
    b.b = GemmOperand{{h, h}, F8, T};
    b.m = D; b.n = F8;
    b.runs = 1;
    out(b, g->dw_down, g->ld_dw_down, F);
    grad(b, g);

    GemmCall &e = second.call[2];          // dWg, dWu
    e.a = GemmOperand{{d, d}, 2 * F8, T};
    e.b = GemmOperand{{x.p, x.p}, x.ld, T};
    e.m = 2 * F8; e.n = x.cols;
    e.runs = 1;
    out(e, g->dw_gate, g->ld_dw_gate, D);
    e.c[1] = g->dw_up;
    e.m_first = F8; e.m_real = F;
    grad(e, g);
    launch(GEMM_BACK, second);
  }

  void grad(GemmCall &c, const chm_ffn_gradients *g) {
    c.f32_out = g->grad_dtype == CHM_F32;
    c.accumulate = g->accumulate != 0;
  }
};

bool aligned(const void *p, int64_t to) { return (uintptr_t)p % to == 0; }

int check(const chm_ffn *f) {
  if (!f || (f->dtype != CHM_BF16 && f->dtype != CHM_F16) || f->activation < CHM_ACT_SILU || f->activation > CHM_ACT_GELU_TANH)
    return CHM_ERR_ARG;
  if (f->tokens < 0 || f->tokens > INT32_MAX || f->width < 1 || f->width > (1 << 24) || f->features < 1 || f->features > (1 << 24)) return CHM_ERR_ARG;
  if (f->ld_x < f->width || f->ld_gate < f->width || f->ld_up < f->width || f->ld_down < f->features) return CHM_ERR_ARG;
  if (f->ld_x > INT32_MAX || f->ld_gate > INT32_MAX || f->ld_up > INT32_MAX || f->ld_down > INT32_MAX) return CHM_ERR_ARG;
  if (!aligned(f->x, 2) || !aligned(f->w_gate, 2) || !aligned(f->w_up, 2) || !aligned(f->w_down, 2) || !aligned(f->saved, 16)) return CHM_ERR_ARG;
  return CHM_OK;
}

using chm_overlap::Rows;
using chm_overlap::stretch;
Rows rows_of(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size) { return Rows{p, rows, cols * size, ld * size}; }

// y is stored when x has been read for the last time: it may lie over x, but over nothing else
bool clash_forward(const chm_ffn *f, void *y, int64_t ld_y, void *scratch, uint64_t scratch_bytes) {
  const int64_t T = f->tokens, D = f->width, F = f->features;
  const Rows x = rows_of(f->x, T, D, f->ld_x, 2), wg = rows_of(f->w_gate, F, D, f->ld_gate, 2), wu = rows_of(f->w_up, F, D, f->ld_up, 2),
             wd = rows_of(f->w_down, D, F, f->ld_down, 2);
  const Rows last[] = {rows_of(y, T, D, ld_y, 2)}, weights[] = {wg, wu, wd};
  const Rows before[] = {stretch(f->saved, f->saved ? (int64_t)kept_bytes(f) : 0), stretch(scratch, (int64_t)scratch_bytes)},
             all[] = {wg, wu, wd, x, last[0]};
  return chm_overlap::clash(last, weights) || chm_overlap::clash(before, all);
}

bool clash_backward(const chm_ffn *f, const chm_ffn_gradients *g, void *scratch, uint64_t scratch_bytes) {
  const int64_t T = f->tokens, D = f->width, F = f->features, size = g->grad_dtype == CHM_F32 ? 4 : 2;
  const int64_t there = T > 0;               // without tokens no input is read
  const Rows results[] = {rows_of(g->dx, T, D, g->ld_dx, 2), rows_of(g->dw_gate, F, D, g->ld_dw_gate, size), rows_of(g->dw_up, F, D, g->ld_dw_up, size),
                          rows_of(g->dw_down, D, F, g->ld_dw_down, size), stretch(scratch, (int64_t)scratch_bytes)};
  const Rows inputs[] = {rows_of(f->x, T, D, f->ld_x, 2), rows_of(g->dy, T, D, g->ld_dy, 2), rows_of(f->w_gate, F * there, D, f->ld_gate, 2),
                         rows_of(f->w_up, F * there, D, f->ld_up, 2), rows_of(f->w_down, D * there, F, f->ld_down, 2), stretch(f->saved, (int64_t)kept_bytes(f))};
  return chm_overlap::clash(results, inputs);
}

// The tiles take rows up to GEMM_LD_MAX elements, dg and du lie side by side in one; the kernels for few tokens count in 64 bits.
bool in_reach(const chm_ffn *f, bool backward) {
  if (f->tokens == 0 || (f->width <= GEMM_LD_MAX && f->features <= GEMM_LD_MAX / 2)) return true;
  return !backward && takes_few(f);
}

int check_gradients(const chm_ffn *f, const chm_ffn_gradients *g) {
  if (!g || (g->grad_dtype != f->dtype && g->grad_dtype != CHM_F32)) return CHM_ERR_ARG;
  const int64_t size = g->grad_dtype == CHM_F32 ? 4 : 2;
  if (g->ld_dy < f->width || g->ld_dx < f->width || g->ld_dw_gate < f->width || g->ld_dw_up != g->ld_dw_gate || g->ld_dw_down < f->features)
    return CHM_ERR_ARG;
  if (g->ld_dy > INT32_MAX || g->ld_dx > INT32_MAX || g->ld_dw_gate > INT32_MAX || g->ld_dw_down > INT32_MAX) return CHM_ERR_ARG;
  if (!aligned(g->dy, 2) || !aligned(g->dx, 2) || !aligned(g->dw_gate, size) || !aligned(g->dw_up, size) || !aligned(g->dw_down, size)) return CHM_ERR_ARG;
  return CHM_OK;
}

}  // namespace

extern "C" int chm_ffn_sizes(const chm_ffn *f, const chm_ffn_gradients *g, uint64_t *saved, uint64_t *forward_scratch, uint64_t *backward_scratch) {
  const int rc = check(f);
  if (rc != CHM_OK) return rc;
  if (g && check_gradients(f, g) != CHM_OK) return CHM_ERR_ARG;
  if ((forward_scratch && !in_reach(f, false)) || (g && !in_reach(f, true))) return CHM_ERR_ARG;
  if (saved) *saved = kept_bytes(f);
  if (forward_scratch) {
    Pass p(f, nullptr, nullptr, false);
    p.forward(nullptr, f->width);
    *forward_scratch = p.arena.used;
  }
  if (backward_scratch) {
    *backward_scratch = 0;
    if (!g) return CHM_OK;
    Pass p(f, nullptr, nullptr, false);
    p.backward(g);
    *backward_scratch = p.arena.used;
  }
  return CHM_OK;
}

extern "C" int chm_ffn_selection(const chm_ffn *f, const chm_ffn_gradients *g, chm_ffn_kernels *out) {
  if (!out || check(f) != CHM_OK || (g && check_gradients(f, g) != CHM_OK) || !in_reach(f, false) || (g && !in_reach(f, true))) return CHM_ERR_ARG;
  Pass p(f, nullptr, nullptr, false);
  p.forward(nullptr, f->width);
  if (g) p.backward(g);
  if (!p.fits) return CHM_ERR_ARG;
  *out = p.chosen;
  return CHM_OK;
}

extern "C" int chm_ffn_forward(const chm_ffn *f, void *y, int64_t ld_y, void *scratch, uint64_t scratch_bytes, void *hip_stream) {
  int rc = check(f);
  if (rc != CHM_OK) return rc;
  if (ld_y < f->width || ld_y > INT32_MAX || !aligned(y, 2) || !aligned(scratch, 16) || !in_reach(f, false)) return CHM_ERR_ARG;
  if (f->tokens == 0) return CHM_OK;
  if (!f->x || !f->w_gate || !f->w_up || !f->w_down || !y || !scratch) return CHM_ERR_ARG;
  Pass need(f, nullptr, nullptr, false);
  need.forward(y, ld_y);
  if (!need.fits) return CHM_ERR_ARG;
  if (scratch_bytes < need.arena.used) return CHM_ERR_LIMIT;
  if (clash_forward(f, y, ld_y, scratch, need.arena.used)) return CHM_ERR_ARG;
  Pass p(f, (char *)scratch, (hipStream_t)hip_stream, true);
  p.forward(y, ld_y);
  return p.ok ? CHM_OK : CHM_ERR_HIP;
}

extern "C" int chm_ffn_backward(const chm_ffn *f, const chm_ffn_gradients *g, void *scratch, uint64_t scratch_bytes, void *hip_stream) {
  int rc = check(f);
  if (rc == CHM_OK) rc = check_gradients(f, g);
  if (rc != CHM_OK) return rc;
  if (!aligned(scratch, 16) || !g->dw_gate || !g->dw_up || !g->dw_down || !in_reach(f, true)) return CHM_ERR_ARG;
  if (f->tokens == 0 && g->accumulate) return CHM_OK;
  if (f->tokens > 0 && (!f->x || !f->w_gate || !f->w_up || !f->w_down || !f->saved || !g->dy || !g->dx || !scratch)) return CHM_ERR_ARG;
  Pass need(f, nullptr, nullptr, false);
  need.backward(g);
  if (!need.fits) return CHM_ERR_ARG;
  if (scratch_bytes < need.arena.used) return CHM_ERR_LIMIT;
  if (clash_backward(f, g, scratch, need.arena.used)) return CHM_ERR_ARG;
  Pass p(f, (char *)scratch, (hipStream_t)hip_stream, true);
  p.backward(g);
  return p.ok ? CHM_OK : CHM_ERR_HIP;
}

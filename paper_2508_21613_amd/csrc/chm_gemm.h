// Matrix products of the gated feed-forward block on the matrix cores: one tile kernel, C[m, n] = sum_k A[m, k] B[n, k],
// for every product of the block's forward and backward pass.
//
// An operand lies in memory with its sums' index k contiguous ("rows": x, h, dy, and the weights in the forward pass) or with
// its own index contiguous ("columns": a weight whose product runs over its other index, both operands of a weight's
// gradient).  Rows go to shared memory as they are and are read 16 bytes a lane; columns go there as they are, too, and are
// transposed on the way to the registers by the LDS transpose reads, so that no transposed copy of anything is made.
// Tiles travel from memory to shared memory without passing through registers; what lies outside an operand arrives as zero
// by the range check of its buffer descriptor, so that odd sizes cost no branch in the loop.
//
// Bank conflicts: the 16-byte chunks of a tile row are stored at chunk ^ f(row); f is chosen per operand such that the 16 lanes
// that read together touch different banks.  The direct loads write linearly, so the permutation is made on their source addresses.
//
// The first operand of a matrix instruction is the n side, the second the m side: a lane then holds four consecutive n of one
// m.  At the end every wavefront turns its sums round in shared memory, 64 rows of 64 at a time, so that a lane goes on with eight
// consecutive n and a row's 64 leave (or meet what they are combined with) as one stretch of memory.  In the two-weight product
// every 16 rows of the gate's weight are followed by the same rows of the up projection's: a wavefront holds both for 32 features.
//
// Sums are float32 (the matrix instructions' accumulators) in one fixed order: results do not change from call to call.
#ifndef CHM_GEMM_H
#define CHM_GEMM_H
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "chm_ffn.h"

namespace chm_gemm {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

struct Bf16 {
  static __device__ __forceinline__ f4 mfma(s8 a, s8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
  static __device__ __forceinline__ float up(uint16_t u) { return __builtin_bit_cast(float, (uint32_t)u << 16); }
};
struct F16 {
  static __device__ __forceinline__ f4 mfma(s8 a, s8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
  static __device__ __forceinline__ float up(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
};

// the activation of g and its derivative, in float32; the reciprocal instruction is right to one unit in the last place.
// Phi(g) = erfc(-g / sqrt 2) / 2: 1 + erf(g / sqrt 2) would cancel to the left of 0 (a tenth of the value at g = -5, all of it from -5.5 on).
template <int ACT> __device__ __forceinline__ float act_of(float g) {
  if (ACT == CHM_ACT_SILU) return g * __builtin_amdgcn_rcpf(1.f + __expf(-g));
  if (ACT == CHM_ACT_GELU) return 0.5f * g * erfcf(g * -0.70710678118654752f);
  // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
  const float z = 0.79788456080286536f * (g + 0.044715f * g * g * g);
  return g * __builtin_amdgcn_rcpf(1.f + __expf(-2.f * z));
}
template <int ACT> __device__ __forceinline__ void act_grad_of(float g, float &a, float &da) {
  if (ACT == CHM_ACT_SILU) {
    const float s = __builtin_amdgcn_rcpf(1.f + __expf(-g));
    a = g * s;
    da = s * (1.f + g * (1.f - s));
  } else if (ACT == CHM_ACT_GELU) {
    const float p = 0.5f * erfcf(g * -0.70710678118654752f);
    a = g * p;
    da = p + g * 0.39894228040143268f * __expf(-0.5f * g * g);
  } else {
    const float z = 0.79788456080286536f * (g + 0.044715f * g * g * g);
    const float s = __builtin_amdgcn_rcpf(1.f + __expf(-2.f * z));
    a = g * s;
    da = s + 2.f * g * s * (1.f - s) * 0.79788456080286536f * (1.f + 3.f * 0.044715f * g * g);
  }
}

enum { ROWS = 0, COLS = 1 };                       // k contiguous / own index contiguous
enum { EPI_STORE = 0, EPI_ACT = 1, EPI_ACT_GRAD = 2 };
enum { BK = 64 };                                  // sums of a step
enum { TURN_ROW = 272 };                           // bytes of 64 float32 and a gap that spreads the rows over the banks

__device__ __forceinline__ uint32_t swz_rows(uint32_t row) { return row & 7u; }
// W: the indices of a row; rows of 64 take half the banks, two of them all
template <int W> __device__ __forceinline__ uint32_t swz_cols(uint32_t k) {
  return W == 64 ? (k & 2u) | (((k >> 3) & 1u) << 2) : ((k & 3u) << 1) | (((k >> 3) & 1u) << 3);
}

// One operand's way from memory to shared memory: W of its indices x BK sums a step, by NT threads.
template <int KIND, int DUAL, int W, int NT>
struct Feed {
  enum : uint32_t { OUT = 0x7fffffff };
  enum { CHUNKS = BK / 8, NI = W * BK * 2 / 16 / NT, BYTES = W * BK * 2 };
  static_assert((W - 1) * GEMM_LD_MAX * 2 + BK * 2 <= OUT && (BK - 1) * GEMM_LD_MAX * 2 + W * 2 <= OUT, "offsets within a tile");
  const char *base;        // of the tile at the present step
  const char *base2;       // of the tile at the second run of k
  int64_t step_bytes;      // from one step to the next
  uint32_t ld_bytes;       // from one row of memory to the next
  uint32_t rows;           // ROWS: rows of the tile less one; COLS: bytes of a row from the tile's first index to the operand's edge
  int32_t k_left;          // sums from the present step's first to the end of the run of k; below 1: nothing is left
  uint32_t off[NI];

  // at: first index of the tile, size: the operand's indices, from sum k0 of the run `seg` on.  wave: uniform.  Two weights side by side:
  // rows 16 to 31 of every 32 are the second's; the rows of one wavefront's loads belong to one of them.
  __device__ __forceinline__ void start(const GemmOperand &o, int64_t at, int64_t size, int seg, int64_t k0, int wave, int tid) {
    ld_bytes = (uint32_t)(o.ld * 2);
    const char *p = (const char *)(DUAL ? o.p[(wave >> 1) & 1] : o.p[seg]);
    const int64_t along = KIND == ROWS ? 2 : o.ld * 2, across = KIND == ROWS ? o.ld * 2 : 2;
    base = p + at * across + k0 * along;
    base2 = (const char *)o.p[1] + at * across;
    step_bytes = along * BK;
    k_left = (int32_t)(o.k - k0);
    if (KIND == ROWS) {
      const int64_t cap = DUAL ? W / 2 : W, n = size - at;
      rows = (uint32_t)(n < cap ? n : cap) - 1;
    } else {
      const int64_t w = (((size + 7) & ~(int64_t)7) - at) * 2;      // whole words of 8: an operand that has no such rows is packed
      rows = (uint32_t)(w < W * 2 ? w : W * 2);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t idx = i * NT + tid;
      if (KIND == ROWS) {
        const uint32_t row = idx / CHUNKS, r = DUAL ? (row >> 5) * 16 + (row & 15u) : row;
        off[i] = r * ld_bytes + chunk_of(i, tid) * 16;
      } else {
        const uint32_t k = idx / (W / 8), chunk = (idx % (W / 8)) ^ swz_cols<W>(k);
        off[i] = chunk * 16 >= rows ? OUT : k * ld_bytes + chunk * 16;
      }
    }
  }
  __device__ __forceinline__ static uint32_t chunk_of(int i, int tid) {
    const uint32_t idx = i * NT + tid;
    return (idx % CHUNKS) ^ swz_rows(idx / CHUNKS);
  }
  // the second run of k begins
  __device__ __forceinline__ void turn(const GemmOperand &o) {
    base = base2;
    k_left = (int32_t)o.k;
  }
  // a step's loads, one by one
  i4 rsrc;                 // buffer descriptor: base, bytes from there to the end of the last element that is there, raw 32-bit words
  uint32_t offset[NI];
  __device__ __forceinline__ void begin(int tid) {
    const uint64_t at = (uint64_t)base;
    rsrc[0] = (int)(uint32_t)at;
    rsrc[1] = (int)(uint32_t)(at >> 32) & 0xffff;
    rsrc[3] = 0x00027000;
    if (k_left >= BK) {
      rsrc[2] = (int)(KIND == ROWS ? rows * ld_bytes + BK * 2 : (BK - 1) * ld_bytes + rows);
#pragma unroll
      for (int i = 0; i < NI; ++i) offset[i] = off[i];
    } else {
      const int32_t left = __builtin_amdgcn_readfirstlane(k_left < 0 ? 0 : k_left);
      rsrc[2] = left > 0 ? (int)(KIND == ROWS ? rows * ld_bytes + left * 2 : (left - 1) * ld_bytes + rows) : 0;
#pragma unroll
      for (int i = 0; i < NI; ++i) offset[i] = KIND == ROWS && (int32_t)chunk_of(i, tid) * 8 >= left ? (uint32_t)OUT : off[i];
    }
    base += step_bytes;
    k_left -= BK;
  }
  // Written out, because the compiler otherwise waits for all loads under way before every transposing read of shared memory.  It writes no
  // register; the waits for what it brings are in arrived().
  __device__ __forceinline__ void one(int i, uint32_t lds, int wave) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset[i]), "s"(rsrc), "s"(lds + (i * NT + wave * 64) * 16));
  }
};

// 8 sums (of the 32 `ks`) of one index of the 16 from `first` on, from the tile in shared memory
template <int KIND, int W>
__device__ __forceinline__ s8 fragment(const lds_char *lds, int first, int ks, int lane) {
  const uint32_t q = lane >> 4, c = lane & 15;
  if (KIND == ROWS) {
    const uint32_t row = first + c, chunk = (ks * 4 + q) ^ swz_rows(row);
    return *(const __attribute__((address_space(3))) s8 *)(lds + row * (BK * 2) + chunk * 16);
  }
  s4 half[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t k = ks * 32 + q * 8 + h * 4 + (c >> 2), chunk = (first / 8 + ((c & 3) >> 1)) ^ swz_cols<W>(k);
    half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(lds + k * (W * 2) + chunk * 16 + (c & 1) * 8));
  }
  return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// The fragments of 32 sums of a wavefront's 16 MT x 64 part of the tile
template <int A_KIND, int B_KIND, int TM, int TN, int MT>
struct Fragments {
  enum { READS = MT + 4 };
  s8 a[MT], b[4];
  // the i-th of READS fragments
  __device__ __forceinline__ void read(int i, const lds_char *ta, const lds_char *tb, int wm, int wn, int ks, int lane) {
    if (i < 4) b[i & 3] = fragment<B_KIND, TN>(tb, wn + i * 16, ks, lane);
    else a[(i - 4) & (MT - 1)] = fragment<A_KIND, TM>(ta, wm + (i - 4) * 16, ks, lane);
  }
};

// Tile and part of the sums of workgroup `block` of a call; false: there is none (a call's workgroups are made a multiple of 8).  Consecutive
// tiles of one die (workgroups go round the 8 dies) share operands in its cache, in bands of 8 tiles along m.
__device__ __forceinline__ bool tile_of(const GemmCall &c, int block, int &tm, int &tn, int &split) {
  const int n = c.tiles_m * c.tiles_n, padded = (n + 7) & ~7;
  split = block / padded;
  block -= split * padded;
  const int die = block & 7, i = block >> 3, per = n >> 3, rem = n & 7;
  if (i >= per + (die < rem)) return false;
  const int t = die * per + (die < rem ? die : rem) + i;
  const int band = 8 * c.tiles_n, b = t / band, r = t - b * band;
  const int rows = c.tiles_m - b * 8 < 8 ? c.tiles_m - b * 8 : 8;
  tm = b * 8 + r % rows;
  tn = r / rows;
  return true;
}

template <class T> __device__ __forceinline__ s8 pack8(const float *v) {
  s8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (short)T::down(v[i]);
  return r;
}

// What large products store for the caller or for much later goes past the caches (PAST), where it would displace the operands: a step of 4,096
// tokens, 4,096 x 11,008, takes 2,754 us with and 2,818 without.  What the next launch reads (h, the gradients of the projections) is better left
// there.
#define CHM_PUT(p, v) do { if (PAST) __builtin_nontemporal_store(v, p); else *(p) = v; } while (0)

// Eight values of row m from column n on: part of a split sum, or a plain output
template <class T, int PAST>
__device__ __forceinline__ void finish_plain(const GemmCall &c, int split, int64_t m, int64_t n, const f4 *v) {
  if (m >= c.m || n >= c.n) return;
  if (c.splits > 1) {
    float *p = c.part + ((int64_t)split * c.m + m) * c.ld_part + n;
    *(f4 *)p = v[0];
    *(f4 *)(p + 4) = v[1];
    return;
  }
  const int which = m >= c.m_first;
  const int64_t row = m - (which ? c.m_first : 0), left = c.n_real - n;
  if (row >= c.m_real || left <= 0) return;
  const bool whole = left >= 8;             // outputs start on any element: 16-byte accesses at any address
  if (c.f32_out) {
    typedef f4 f4_anywhere __attribute__((aligned(4)));
    float *p = (float *)c.c[which] + row * c.ldc + n;
    if (whole) {
      f4 a = v[0], b = v[1];
      if (c.accumulate) { a += *(const f4_anywhere *)p; b += *(const f4_anywhere *)(p + 4); }
      CHM_PUT((f4_anywhere *)p, a);
      CHM_PUT((f4_anywhere *)(p + 4), b);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) p[e] = c.accumulate ? v[e >> 2][e & 3] + p[e] : v[e >> 2][e & 3];
    }
    return;
  }
  typedef s8 s8_anywhere __attribute__((aligned(2)));
  uint16_t *p = (uint16_t *)c.c[which] + row * c.ldc + n;
  float w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = v[e >> 2][e & 3];
  if (whole) {
    if (c.accumulate) {
      const s8 old = *(const s8_anywhere *)p;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += T::up((uint16_t)old[e]);
    }
    CHM_PUT((s8_anywhere *)p, pack8<T>(w));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = T::down(c.accumulate ? w[e] + T::up(p[e]) : w[e]);
  }
}

// Values kept for the backward pass: the upper 24 bits of float32 (16 of them significant), 1.5 times the bytes of the tensors' own type.
// Rounded to that type they would add an error as large as all others together to every gradient.  Rounded to the nearest, half away from
// zero: cut off they are too small by 2^-17 to 2^-16 on average, which a float32 gradient over 65,536 tokens shows (1.3e-5 to 2.7e-5 of itself,
// ten times its other errors).  Infinities stay, and so does what is not a number: sums of products of 16-bit values have zeros in its lower bits.
//
// They lie in blocks of 16 rows x 32 features of 3 KiB: upper 16 bits of g, those of u, lower 8 of both, each eight features' 16 bytes behind
// the other, row by row.  That is how the 64 lanes of a wavefront hold them: every store is one stretch of 1 KiB (in planes of rows
// they were pieces of 64 and 32 bytes, and cost twice the time that their bytes take).
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ char *kept_at(const Kept &k, int64_t m, int64_t f) {
  return k.p + ((m >> 4) * k.blocks + (f >> 5)) * 3072 + ((m & 15) * 4 + ((f >> 3) & 3)) * 16;
}
__device__ __forceinline__ uint32_t upper24(float v) { return __float_as_uint(v) + 0x80u; }      // in the upper 24 bits; the others are left over
template <int PAST>
__device__ __forceinline__ void keep8(const Kept &k, int64_t m, int64_t f, const float *g, const float *u) {
  u4 hi[2], lo;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = upper24(w ? u[e] : g[e]);
#pragma unroll
    for (int i = 0; i < 4; ++i) hi[w][i] = __builtin_amdgcn_perm(v[2 * i + 1], v[2 * i], 0x07060302);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      lo[w * 2 + i] = __builtin_amdgcn_perm(v[4 * i + 1], v[4 * i], 0x0c0c0501) | __builtin_amdgcn_perm(v[4 * i + 3], v[4 * i + 2], 0x05010c0c);
  }
  char *p = kept_at(k, m, f);
  CHM_PUT((u4 *)p, hi[0]);
  CHM_PUT((u4 *)(p + 1024), hi[1]);
  CHM_PUT((u4 *)(p + 2048), lo);
}
struct Kept8 { u4 g, u, lo; };
__device__ __forceinline__ Kept8 kept8(const Kept &k, int64_t m, int64_t f) {
  const char *p = kept_at(k, m, f);
  return Kept8{__builtin_nontemporal_load((const u4 *)p), __builtin_nontemporal_load((const u4 *)(p + 1024)), __builtin_nontemporal_load((const u4 *)(p + 2048))};
}
__device__ __forceinline__ void unkeep8(u4 hi, u2 lo, float *v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // bytes from the top: upper 16 bits of the value, its lower 8, zero
    const uint32_t sel = (e & 1 ? 0x07060000u : 0x05040000u) | ((uint32_t)(e & 3) << 8) | 0x0cu;
    v[e] = __uint_as_float(__builtin_amdgcn_perm(hi[e >> 1], lo[e >> 2], sel));
  }
}

// Eight features of both projections (float32 sums): activation and product
template <class T, int ACT, int PAST>
__device__ __forceinline__ void finish_pair(const GemmCall &c, int64_t m, int64_t f, const f4 *v) {
  if (m >= c.m || f >= c.n) return;
  float g[8], u[8], h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    g[e] = v[e >> 2][e & 3];
    u[e] = v[2 + (e >> 2)][e & 3];
    h[e] = act_of<ACT>(g[e]) * u[e];
  }
  if (f + 8 > c.n) {                        // rows are whole words of 8, zeros behind the features
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (f + e >= c.n) g[e] = u[e] = h[e] = 0.f;
  }
  const int64_t at = m * c.ldi + f;
  *(s8 *)(c.h + at) = pack8<T>(h);
  if (c.kept.p) keep8<PAST>(c.kept, m, f, g, u);
}

// Eight features of dh: the gradients of both projections, and h
template <class T, int ACT>
__device__ __forceinline__ void finish_gradient(const GemmCall &c, int64_t m, int64_t f, const f4 *v, const Kept8 &k) {
  if (m >= c.m || f >= c.n) return;
  float g[8], u[8], h[8], dg[8], du[8];
  unkeep8(k.g, u2{k.lo[0], k.lo[1]}, g);
  unkeep8(k.u, u2{k.lo[2], k.lo[3]}, u);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float dh = v[e >> 2][e & 3];
    float a, da;
    act_grad_of<ACT>(g[e], a, da);
    h[e] = a * u[e];
    du[e] = dh * a;
    dg[e] = dh * u[e] * da;
  }
  if (f + 8 > c.n_real) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (f + e >= c.n_real) h[e] = du[e] = dg[e] = 0.f;
  }
  *(s8 *)(c.h + m * c.ldi + f) = pack8<T>(h);
  *(s8 *)(c.dgate + m * c.ldd + f) = pack8<T>(dg);
  *(s8 *)(c.dup + m * c.ldd + f) = pack8<T>(du);
}

typedef __attribute__((address_space(3))) f4 lds_f4;

// A wavefront's ROWS_ rows of 64 sums, turned round in shared memory at `turn`; m1, n1: the first row and column (feature) of them.
// A loop, not a sequence: code that runs once a tile is read from the cache of instructions' own source, and slowly.
template <class T, int DUAL, int EPI, int ACT, int ROWS_, int PAST>
__device__ __forceinline__ void finish(const GemmCall &c, int split, const lds_char *turn, int64_t m1, int64_t n1, int lane) {
  if (DUAL) {                               // 16 rows of 32 features at a time
    const int f = (lane & 3) * 8;
#pragma nounroll
    for (int r = lane >> 2; r < ROWS_; r += 16) {
      const lds_char *at = turn + r * TURN_ROW + ((f >> 4) * 32 + (f & 8)) * 4;
      const f4 v[4] = {*(const lds_f4 *)at, *(const lds_f4 *)(at + 16), *(const lds_f4 *)(at + 64), *(const lds_f4 *)(at + 80)};
      finish_pair<T, ACT, PAST>(c, m1 + r, n1 + f, v);
    }
    return;
  }
  // 8 rows of 64 at a time
  const int64_t n = n1 + (lane & 7) * 8;
  const lds_char *at = turn + (lane >> 3) * TURN_ROW + (lane & 7) * 32;
  int64_t m = m1 + (lane >> 3);
  if (EPI == EPI_ACT_GRAD) {                // what is kept of two times 8 rows is on its way
    const int64_t col = n < c.n ? n : 0, last = c.m - 1;
    Kept8 kept[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) kept[i] = kept8(c.kept, m + i * 8 < last ? m + i * 8 : last, col);
#pragma nounroll
    for (int r = 0; r < ROWS_; r += 16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const Kept8 k = kept[i];
        kept[i] = kept8(c.kept, m + 16 < last ? m + 16 : last, col);
        const f4 v[2] = {*(const lds_f4 *)at, *(const lds_f4 *)(at + 16)};
        finish_gradient<T, ACT>(c, m, n, v, k);
        at += 8 * TURN_ROW;
        m += 8;
      }
    }
    return;
  }
#pragma nounroll
  for (int r = 0; r < ROWS_; r += 8) {
    const f4 v[2] = {*(const lds_f4 *)at, *(const lds_f4 *)(at + 16)};
    finish_plain<T, PAST>(c, split, m, n, v);
    at += 8 * TURN_ROW;
    m += 8;
  }
}

// Both operands of a step, into one of the slots in shared memory; behind the last step zeros arrive: the number of loads under way
// is the same in every step
template <class FeedA, class FeedB>
struct Fetch {
  const GemmCall &c;
  FeedA a;
  FeedB b;
  int turn_at, wave, tid;
  uint32_t lds;
  enum { LOADS = FeedA::NI + FeedB::NI, A_BYTES = FeedA::BYTES, STAGE = FeedA::BYTES + FeedB::BYTES };
  __device__ __forceinline__ void begin(int step) {
    if (step == turn_at) {
      a.turn(c.a);
      b.turn(c.b);
    }
    a.begin(tid);
    b.begin(tid);
  }
  __device__ __forceinline__ void one(int i, int slot) {
    if (i < FeedA::NI) a.one(i, lds + slot * STAGE, wave);
    else b.one(i - FeedA::NI, lds + slot * STAGE + A_BYTES, wave);
  }
};

// waits until at most PENDING loads are under way and all shared memory reads are back, then for the workgroup
template <int PENDING>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PENDING) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 4 MT matrix instructions on the fragments `now`; between them the fragments `next` are read (from `from`, its sums `ks`) and, with
// LOAD, the loads of a later step are issued into `slot`
template <class T, int MT, int LOAD, class F, class G>
__device__ __forceinline__ void multiply(const F &now, F &next, f4 (&acc)[4][MT], G &fetch, int slot, const lds_char *from, int ks, int wm, int wn, int lane) {
  constexpr int M = 4 * MT, LOADS = LOAD ? G::LOADS : 0, READS = F::READS;
#pragma unroll
  for (int i = 0; i < M; ++i) {
#pragma unroll
    for (int l = i * LOADS / M; l < (i + 1) * LOADS / M; ++l) fetch.one(l, slot);
#pragma unroll
    for (int r = i * READS / M; r < (i + 1) * READS / M; ++r) next.read(r, from, from + G::A_BYTES, wm, wn, ks, lane);
    acc[i & 3][i >> 2] = T::mfma(now.b[i & 3], now.a[i >> 2], acc[i & 3][i >> 2]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// bytes of shared memory of a configuration: the steps under way, or the sums that are turned round at the end
template <int WM, int WN, int MT, int SLOTS> constexpr int shared_bytes() {
  constexpr int stage = (WM * MT * 16 + WN * 64) * BK * 2, turn = WM * WN * (MT < 4 ? MT * 16 : 64) * TURN_ROW;
  return SLOTS * stage > turn ? SLOTS * stage : turn;
}

// One tile of one product
template <class T, int A_KIND, int B_KIND, int DUAL, int EPI, int WM, int WN, int MT, int SLOTS>
__device__ __forceinline__ void tile_product(const GemmCall &c, int block, lds_char *lds) {
  constexpr int NT = 64 * WM * WN, TM = WM * MT * 16, TN = WN * 64;
  typedef Feed<A_KIND, 0, TM, NT> FeedA;
  typedef Feed<B_KIND, DUAL, TN, NT> FeedB;
  typedef Fragments<A_KIND, B_KIND, TM, TN, MT> Frags;
  constexpr int STAGE = FeedA::BYTES + FeedB::BYTES, LOADS = FeedA::NI + FeedB::NI;
  constexpr int TURN = MT < 4 ? MT * 16 : 64;        // rows turned round at a time
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tm, tn, split;
  if (!tile_of(c, block, tm, tn, split)) return;
  const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * (DUAL ? TN / 2 : TN);
  const int wm = (wave / WN) * (MT * 16), wn = (wave % WN) * 64;

  // steps of this workgroup
  const int steps_seg = (int)(((c.a.k > c.b.k ? c.a.k : c.b.k) + BK - 1) / BK), steps = steps_seg * c.runs;
  int step = 0, last = steps;
  if (c.splits > 1) {
    step = (int)((int64_t)steps * split / c.splits);
    last = (int)((int64_t)steps * (split + 1) / c.splits);
  }
  Fetch<FeedA, FeedB> fetch{c, {}, {}, c.runs > 1 ? steps_seg : -1, wave, tid, (uint32_t)(uintptr_t)lds};
  const int seg = c.runs > 1 && step >= steps_seg;
  const int64_t k0 = (int64_t)(step - seg * steps_seg) * BK;
  fetch.a.start(c.a, m0, c.m, seg, k0, wave, tid);
  fetch.b.start(c.b, n0, c.n, seg, k0, wave, tid);

  f4 acc[4][MT];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[j][t] = f4{0.f, 0.f, 0.f, 0.f};

  // SLOTS buffers in shared memory, two sets of fragments in registers.  While the matrix instructions of 32 sums run, the
  // fragments of the next 32 are read, and in a step's second half the loads of the step SLOTS ahead are issued: all of them
  // spread between the matrix instructions, which they would hold up if they were issued in a row.  One barrier a step: behind it
  // the next step's tiles have arrived, and the present ones have been read by everybody.
  Frags even, odd;
  if (step < last) {
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      fetch.begin(step + i);
#pragma unroll
      for (int l = 0; l < LOADS; ++l) fetch.one(l, i);
    }
    arrived<(SLOTS - 1) * LOADS>();
#pragma unroll
    for (int i = 0; i < Frags::READS; ++i) even.read(i, lds, lds + FeedA::BYTES, wm, wn, 0, lane);
  }
  for (int slot = 0; step < last; ++step) {
    multiply<T, MT, 0>(even, odd, acc, fetch, slot, lds + slot * STAGE, 1, wm, wn, lane);
    fetch.begin(step + SLOTS);
    arrived<(SLOTS - 2) * LOADS>();
    const int next = slot + 1 == SLOTS ? 0 : slot + 1;
    multiply<T, MT, 1>(odd, even, acc, fetch, slot, lds + next * STAGE, 0, wm, wn, lane);
    slot = next;
  }

  arrived<0>();                             // the tiles are read no more, and nothing is under way to them
  lds_char *turn = lds + wave * (TURN * TURN_ROW);
#pragma unroll
  for (int t0 = 0; t0 < MT; t0 += TURN / 16) {
#pragma unroll
    for (int t = t0; t < t0 + TURN / 16; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) *(lds_f4 *)(turn + ((t - t0) * 16 + (lane & 15)) * TURN_ROW + (j * 16 + (lane >> 4) * 4) * 4) = acc[j][t];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int64_t m1 = m0 + wm + t0 * 16, n1 = n0 + (DUAL ? wn / 2 : wn);
    if (EPI == EPI_STORE || c.act == CHM_ACT_SILU) finish<T, DUAL, EPI, CHM_ACT_SILU, TURN, MT == 8>(c, split, turn, m1, n1, lane);
    else if (c.act == CHM_ACT_GELU) finish<T, DUAL, EPI, CHM_ACT_GELU, TURN, MT == 8>(c, split, turn, m1, n1, lane);
    else finish<T, DUAL, EPI, CHM_ACT_GELU_TANH, TURN, MT == 8>(c, split, turn, m1, n1, lane);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

template <class T, int PRODUCTS, int WM, int WN, int MT, int SLOTS>
__global__ void __launch_bounds__(64 * WM * WN, 1) __attribute__((amdgpu_waves_per_eu(MT == 2 && SLOTS == 2 ? 4 : 2))) k_gemm(const GemmGroup g) {
#ifdef __HIP_DEVICE_COMPILE__        // the host pass knows no instructions of the matrix cores
  __shared__ __attribute__((aligned(1024))) char shared[shared_bytes<WM, WN, MT, SLOTS>()];
  lds_char *lds = (lds_char *)shared;
  const int block = blockIdx.x;
  if (PRODUCTS == GEMM_GATE_UP) tile_product<T, ROWS, ROWS, 1, EPI_ACT, WM, WN, MT, SLOTS>(g.call[0], block, lds);
  else if (PRODUCTS == GEMM_OUT) tile_product<T, ROWS, ROWS, 0, EPI_STORE, WM, WN, MT, SLOTS>(g.call[0], block, lds);
  else if (PRODUCTS == GEMM_DH) tile_product<T, ROWS, COLS, 0, EPI_ACT_GRAD, WM, WN, MT, SLOTS>(g.call[0], block, lds);
  else if (block < g.first[1]) tile_product<T, ROWS, COLS, 0, EPI_STORE, WM, WN, MT, SLOTS>(g.call[0], block, lds);
  else {
    const int i = block < g.first[2] ? 1 : 2;
    tile_product<T, COLS, COLS, 0, EPI_STORE, WM, WN, MT, SLOTS>(g.call[i], block - g.first[i], lds);
  }
#endif
}

template <class T, int PRODUCTS>
bool launch_products(int tile, const GemmGroup &g, hipStream_t st) {
  const dim3 grid((uint32_t)g.first[g.count]);
  if (tile == TILE_256) hipLaunchKernelGGL((k_gemm<T, PRODUCTS, 2, 4, 8, 2>), grid, dim3(512), 0, st, g);
  else if (tile == TILE_128_DEEP) hipLaunchKernelGGL((k_gemm<T, PRODUCTS, 4, 2, 2, 4>), grid, dim3(512), 0, st, g);
  else if (tile == TILE_64 && PRODUCTS != GEMM_BACK) hipLaunchKernelGGL((k_gemm<T, PRODUCTS == GEMM_BACK ? GEMM_OUT : PRODUCTS, 4, 1, 1, 4>), grid, dim3(256), 0, st, g);
  else hipLaunchKernelGGL((k_gemm<T, PRODUCTS, 4, 2, 2, 2>), grid, dim3(512), 0, st, g);
  return hipGetLastError() == hipSuccess;
}

template <class T>
bool launch(int products, int tile, const GemmGroup &g, void *stream) {
  hipStream_t st = (hipStream_t)stream;
  switch (products) {
    case GEMM_GATE_UP: return launch_products<T, GEMM_GATE_UP>(tile, g, st);
    case GEMM_OUT: return launch_products<T, GEMM_OUT>(tile, g, st);
    case GEMM_DH: return launch_products<T, GEMM_DH>(tile, g, st);
    default: return launch_products<T, GEMM_BACK>(tile, g, st);
  }
}

}  // namespace chm_gemm
#endif

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
// m.  At the end every wavefront turns its sums round in shared memory, 32 rows of 64 at a time, so that a lane goes on with eight
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

// the activation of g and its derivative, in float32
__device__ __forceinline__ float act_of(int act, float g) {
  if (act == CHM_ACT_SILU) return g / (1.f + __expf(-g));
  if (act == CHM_ACT_GELU) return 0.5f * g * (1.f + erff(g * 0.70710678118654752f));
  // 0.5 (1 + tanh z) = 1 / (1 + exp(-2 z))
  const float z = 0.79788456080286536f * (g + 0.044715f * g * g * g);
  return g / (1.f + __expf(-2.f * z));
}
__device__ __forceinline__ void act_grad_of(int act, float g, float &a, float &da) {
  if (act == CHM_ACT_SILU) {
    const float s = 1.f / (1.f + __expf(-g));
    a = g * s;
    da = s * (1.f + g * (1.f - s));
  } else if (act == CHM_ACT_GELU) {
    const float p = 0.5f * (1.f + erff(g * 0.70710678118654752f));
    a = g * p;
    da = p + g * 0.39894228040143268f * __expf(-0.5f * g * g);
  } else {
    const float z = 0.79788456080286536f * (g + 0.044715f * g * g * g);
    const float s = 1.f / (1.f + __expf(-2.f * z));
    a = g * s;
    da = s + 2.f * g * s * (1.f - s) * 0.79788456080286536f * (1.f + 3.f * 0.044715f * g * g);
  }
}

enum { ROWS = 0, COLS = 1 };                       // k contiguous / own index contiguous
enum { EPI_STORE = 0, EPI_ACT = 1, EPI_ACT_GRAD = 2 };
enum { BK = 64 };
enum { TURN_ROW = 272 };                           // bytes of 64 float32 and a gap that spreads the rows over the banks

// 24 bits of a float32, rounded to nearest, ties to even; not a number stays one
__device__ __forceinline__ uint32_t keep_bits(float f) {
  const uint32_t b = __float_as_uint(f), r = b + 0x7fu + ((b >> 8) & 1u);
  return f != f ? b | 0x00400000u : r;
}


__device__ __forceinline__ uint32_t swz_rows(uint32_t row) { return row & 7u; }
__device__ __forceinline__ uint32_t swz_cols(uint32_t k) { return ((k & 3u) << 1) | (((k >> 3) & 1u) << 3); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const char *p, int64_t bytes) {
  const uint32_t n = bytes <= 0 ? 0u : bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes;
  return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)n, 0x00027000);
}

// One operand's way from memory to shared memory: W of its indices x BK sums a step, by NT threads.
template <int KIND, int DUAL, int W, int NT>
struct Feed {
  enum : uint32_t { OUT = 0x7fffffff };
  enum { NI = W * BK * 2 / 16 / NT, BYTES = W * BK * 2 };
  const char *base;        // of the tile at the present step
  int64_t ld_bytes;        // from one row of memory to the next
  int64_t left;            // ROWS: bytes from base to the end of the tile's last row
  int64_t k_left;          // sums from the present step's first to the end of the run of k
  int64_t width;           // bytes of a row from the tile's first index to the operand's edge (COLS), rows of the tile (ROWS)
  uint32_t off[NI];

  // at: first index of the tile, size: the operand's indices.  wave: uniform.
  __device__ __forceinline__ void start(const GemmOperand &o, int64_t at, int64_t size, int tid) {
    ld_bytes = o.ld * 2;
    if (KIND == ROWS) {
      const int64_t cap = DUAL ? W / 2 : W, rows = size - at;
      width = rows < cap ? rows : cap;
    } else {
      width = (((size + 7) & ~(int64_t)7) - at) * 2;      // whole words of 8: an operand that has no such rows is packed
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const uint32_t idx = i * NT + tid;
      if (KIND == ROWS) {
        const uint32_t row = idx / 8, chunk = (idx & 7u) ^ swz_rows(row);
        const uint32_t r = DUAL ? (row >> 5) * 16 + (row & 15u) : row;
        off[i] = r * (uint32_t)ld_bytes + chunk * 16;
      } else {
        const uint32_t k = idx / (W / 8), chunk = (idx % (W / 8)) ^ swz_cols(k);
        off[i] = (int64_t)chunk * 16 >= width ? OUT : k * (uint32_t)ld_bytes + chunk * 16;
      }
    }
  }
  // The run of k `seg`, from sum k0 on.  Two weights side by side: rows 16 to 31 of every 32 are the second's; the rows of one
  // wavefront's loads belong to one of them.
  __device__ __forceinline__ void seek(const GemmOperand &o, int64_t at, int seg, int64_t k0, int wave) {
    const char *p = (const char *)(DUAL ? o.p[(wave >> 1) & 1] : o.p[seg]);
    k_left = o.k - k0;
    if (KIND == ROWS) {
      base = p + at * ld_bytes + k0 * 2;
      left = (width - 1) * ld_bytes + (o.k - k0) * 2;
    } else {
      base = p + k0 * ld_bytes + at * 2;
    }
  }
  __device__ __forceinline__ void load(lds_char *lds, int wave, int tid) {
    if (KIND == ROWS) {
      const __amdgpu_buffer_rsrc_t r = rsrc_of(base, left);
      if (k_left >= BK) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds + (i * NT + wave * 64) * 16), 16, off[i], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const uint32_t row = (i * NT + tid) / 8, chunk = (tid & 7u) ^ swz_rows(row);
          const uint32_t v = (int64_t)chunk * 8 >= k_left ? OUT : off[i];
          __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds + (i * NT + wave * 64) * 16), 16, v, 0, 0, 0);
        }
      }
      base += BK * 2;
      left -= BK * 2;
    } else {
      const int64_t rows = k_left < BK ? k_left : BK;
      const __amdgpu_buffer_rsrc_t r = rsrc_of(base, (rows - 1) * ld_bytes + width);
#pragma unroll
      for (int i = 0; i < NI; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds + (i * NT + wave * 64) * 16), 16, off[i], 0, 0, 0);
      base += BK * ld_bytes;
    }
    k_left -= BK;
  }
};

// 8 sums of one index of the 16 from `first` on, from the tile in shared memory
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
    const uint32_t k = ks * 32 + q * 8 + h * 4 + (c >> 2), chunk = (first / 8 + ((c & 3) >> 1)) ^ swz_cols(k);
    half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(lds + k * (W * 2) + chunk * 16 + (c & 1) * 8));
  }
  return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// The fragments of 32 sums of a wavefront's 16 MT x 64 part of the tile
template <int A_KIND, int B_KIND, int TM, int TN, int MT>
struct Fragments {
  enum { READS = (A_KIND == ROWS ? MT : 2 * MT) + (B_KIND == ROWS ? 4 : 8) };
  s8 a[MT], b[4];
  __device__ __forceinline__ void read(const lds_char *ta, const lds_char *tb, int wm, int wn, int ks, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = fragment<B_KIND, TN>(tb, wn + j * 16, ks, lane);
#pragma unroll
    for (int t = 0; t < MT; ++t) a[t] = fragment<A_KIND, TM>(ta, wm + t * 16, ks, lane);
  }
  template <class T> __device__ __forceinline__ void multiply(f4 (&acc)[4][MT]) const {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j][t] = T::mfma(b[j], a[t], acc[j][t]);
  }
};
// reads spread between the matrix instructions
template <int MT, int READS> __device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < READS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 4 * MT / READS > 0 ? 4 * MT / READS : 1, 0);
  }
}

// tile of this workgroup: consecutive tiles of one die (workgroups go round the 8 dies) share operands in its cache, in bands
// of 8 tiles along m
__device__ __forceinline__ void tile_of(const GemmCall &c, int &tm, int &tn) {
  const int n = c.tiles_m * c.tiles_n, die = blockIdx.x & 7, i = blockIdx.x >> 3;
  const int per = n >> 3, rem = n & 7;
  const int t = die * per + (die < rem ? die : rem) + i;
  const int band = 8 * c.tiles_n, b = t / band, r = t - b * band;
  const int rows = c.tiles_m - b * 8 < 8 ? c.tiles_m - b * 8 : 8;
  tm = b * 8 + r % rows;
  tn = r / rows;
}

template <class T> __device__ __forceinline__ s8 pack8(const float *v) {
  s8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (short)T::down(v[i]);
  return r;
}

// Eight values of row m from column n on: part of a split sum, or a plain output
template <class T>
__device__ __forceinline__ void finish_plain(const GemmCall &c, int64_t m, int64_t n, const f4 *v) {
  if (m >= c.m || n >= c.n) return;
  if (c.splits > 1) {
    float *p = c.part + ((int64_t)blockIdx.y * c.m + m) * c.ld_part + n;
    *(f4 *)p = v[0];
    *(f4 *)(p + 4) = v[1];
    return;
  }
  const int which = m >= c.m_first;
  const int64_t row = m - (which ? c.m_first : 0), left = c.n_real - n;
  if (row >= c.m_real || left <= 0) return;
  const bool whole = c.wide && left >= 8;
  if (c.f32_out) {
    float *p = (float *)c.c[which] + row * c.ldc + n;
    if (whole) {
      f4 a = v[0], b = v[1];
      if (c.accumulate) { a += *(const f4 *)p; b += *(const f4 *)(p + 4); }
      *(f4 *)p = a;
      *(f4 *)(p + 4) = b;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) p[e] = c.accumulate ? v[e >> 2][e & 3] + p[e] : v[e >> 2][e & 3];
    }
    return;
  }
  uint16_t *p = (uint16_t *)c.c[which] + row * c.ldc + n;
  float w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = v[e >> 2][e & 3];
  if (whole) {
    if (c.accumulate) {
      const s8 old = *(const s8 *)p;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += T::up((uint16_t)old[e]);
    }
    *(s8 *)p = pack8<T>(w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = T::down(c.accumulate ? w[e] + T::up(p[e]) : w[e]);
  }
}

// Values kept for the backward pass: rounded to 24 bits (16 of them significant), the upper 16 and the lower 8 apart, 1.5 times the bytes of the
// tensors' own type.  Rounded to that type they would add an error as large as all others together to every gradient.
__device__ __forceinline__ void keep8(uint16_t *high, uint8_t *low, int64_t at, const float *v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  s8 hi;
  u2 lo = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t b = keep_bits(v[e]);
    hi[e] = (short)(b >> 16);
    lo[e >> 2] |= ((b >> 8) & 0xffu) << (8 * (e & 3));
  }
  *(s8 *)(high + at) = hi;
  *(u2 *)(low + at) = lo;
}
__device__ __forceinline__ void kept8(const uint16_t *high, const uint8_t *low, int64_t at, float *v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2)));
  const s8 hi = *(const s8 *)(high + at);
  const u2 lo = *(const u2 *)(low + at);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(((uint32_t)(uint16_t)hi[e] << 16) | (((lo[e >> 2] >> (8 * (e & 3))) & 0xffu) << 8));
}

// Eight features of both projections (float32 sums): activation and product
template <class T>
__device__ __forceinline__ void finish_pair(const GemmCall &c, int64_t m, int64_t f, const f4 *v) {
  if (m >= c.m || f >= c.n) return;
  float g[8], u[8], h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    g[e] = v[e >> 2][e & 3];
    u[e] = v[2 + (e >> 2)][e & 3];
    h[e] = act_of(c.act, g[e]) * u[e];
    if (f + e >= c.n) g[e] = u[e] = h[e] = 0.f;        // rows are whole words of 8, zeros behind the features
  }
  *(s8 *)(c.h + m * c.ldi + f) = pack8<T>(h);
  if (c.kept.gate) {
    keep8(c.kept.gate, c.kept.gate_low, m * c.ldi + f, g);
    keep8(c.kept.up, c.kept.up_low, m * c.ldi + f, u);
  }
}

// Eight features of dh: the gradients of both projections, and h
template <class T>
__device__ __forceinline__ void finish_gradient(const GemmCall &c, int64_t m, int64_t f, const f4 *v) {
  if (m >= c.m || f >= c.n) return;
  float g[8], u[8], h[8], dg[8], du[8];
  kept8(c.kept.gate, c.kept.gate_low, m * c.ldi + f, g);
  kept8(c.kept.up, c.kept.up_low, m * c.ldi + f, u);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float dh = v[e >> 2][e & 3];
    float a, da;
    act_grad_of(c.act, g[e], a, da);
    h[e] = a * u[e];
    du[e] = dh * a;
    dg[e] = dh * u[e] * da;
    if (f + e >= c.n_real) h[e] = du[e] = dg[e] = 0.f;
  }
  *(s8 *)(c.h + m * c.ldi + f) = pack8<T>(h);
  *(s8 *)(c.dgate + m * c.ldd + f) = pack8<T>(dg);
  *(s8 *)(c.dup + m * c.ldd + f) = pack8<T>(du);
}

// Both operands of a step, into one of the two buffers
template <class FeedA, class FeedB>
struct Fetch {
  const GemmCall &c;
  FeedA &a;
  FeedB &b;
  int64_t m0, n0;
  int seg, wave, tid;
  lds_char *lds;
  __device__ __forceinline__ void operator()(int step, int buf) {
    if (step == c.steps_seg && step > 0 && seg == 0) {
      seg = 1;
      a.seek(c.a, m0, 1, 0, wave);
      b.seek(c.b, n0, 1, 0, wave);
    }
    lds_char *to = lds + buf * (FeedA::BYTES + FeedB::BYTES);
    a.load(to, wave, tid);
    b.load(to + FeedA::BYTES, wave, tid);
  }
};

template <class T, int A_KIND, int B_KIND, int DUAL, int EPI, int WM, int WN, int MT>
__global__ void __launch_bounds__(64 * WM * WN, 1) __attribute__((amdgpu_waves_per_eu(2, 2))) k_gemm(const GemmCall c) {
#ifdef __HIP_DEVICE_COMPILE__        // the host pass knows no buffer descriptors
  constexpr int NT = 64 * WM * WN, TM = WM * MT * 16, TN = WN * 64;
  typedef Feed<A_KIND, 0, TM, NT> FeedA;
  typedef Feed<B_KIND, DUAL, TN, NT> FeedB;
  __shared__ __attribute__((aligned(1024))) char shared[2 * (FeedA::BYTES + FeedB::BYTES)];
  lds_char *lds = (lds_char *)shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tm, tn;
  tile_of(c, tm, tn);
  const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * (DUAL ? TN / 2 : TN);
  const int wm = (wave / WN) * (MT * 16), wn = (wave % WN) * 64;

  int step = 0, last = c.steps;
  if (c.splits > 1) {
    step = (int)((int64_t)c.steps * blockIdx.y / c.splits);
    last = (int)((int64_t)c.steps * (blockIdx.y + 1) / c.splits);
  }
  FeedA fa;
  FeedB fb;
  fa.start(c.a, m0, c.m, tid);
  fb.start(c.b, n0, c.n, tid);
  int seg = step >= c.steps_seg;
  const int64_t k0 = (int64_t)(step - seg * c.steps_seg) * BK;
  fa.seek(c.a, m0, seg, k0, wave);
  fb.seek(c.b, n0, seg, k0, wave);

  f4 acc[4][MT];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[j][t] = f4{0.f, 0.f, 0.f, 0.f};

  Fetch<FeedA, FeedB> fetch{c, fa, fb, m0, n0, seg, wave, tid, lds};
  // Two buffers in shared memory, two sets of fragments in registers: while the matrix instructions of one half of a step run, the
  // fragments of the next half are read, and the tiles of the step after next are on their way.  One barrier a step: behind
  // it the next tiles have arrived, and nobody reads the present ones any more.
  Fragments<A_KIND, B_KIND, TM, TN, MT> half0, half1;
  const int buffer = FeedA::BYTES + FeedB::BYTES;
  if (step < last) {
    fetch(step, 0);
    __syncthreads();
    if (step + 1 < last) fetch(step + 1, 1);
    half0.read(lds, lds + FeedA::BYTES, wm, wn, 0, lane);
  }
  int buf = 0;
  for (; step < last; ++step, buf ^= 1) {
    const lds_char *now = lds + buf * buffer, *next = lds + (buf ^ 1) * buffer;
    half1.read(now, now + FeedA::BYTES, wm, wn, 1, lane);
    half0.template multiply<T>(acc);
    interleave<MT, Fragments<A_KIND, B_KIND, TM, TN, MT>::READS>();
    __syncthreads();
    if (step + 2 < last) fetch(step + 2, buf);
    half0.read(next, next + FeedA::BYTES, wm, wn, 0, lane);        // behind the last step: stale, and not used
    half1.template multiply<T>(acc);
    interleave<MT, Fragments<A_KIND, B_KIND, TM, TN, MT>::READS>();
  }

  __syncthreads();                          // the tiles are read no more
  typedef __attribute__((address_space(3))) f4 lds_f4;
  lds_char *turn = lds + wave * (32 * TURN_ROW);
#pragma unroll
  for (int t0 = 0; t0 < MT; t0 += 2) {
#pragma unroll
    for (int t = t0; t < t0 + 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) *(lds_f4 *)(turn + ((t - t0) * 16 + (lane & 15)) * TURN_ROW + (j * 16 + (lane >> 4) * 4) * 4) = acc[j][t];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int64_t m1 = m0 + wm + t0 * 16;
    if (DUAL) {
      // 16 rows of 32 features at a time
#pragma nounroll
      for (int r = lane >> 2; r < 32; r += 16) {
        const int f = (lane & 3) * 8;
        const lds_char *at = turn + r * TURN_ROW + ((f >> 4) * 32 + (f & 8)) * 4;
        const f4 v[4] = {*(const lds_f4 *)at, *(const lds_f4 *)(at + 16), *(const lds_f4 *)(at + 64), *(const lds_f4 *)(at + 80)};
        finish_pair<T>(c, m1 + r, n0 + wn / 2 + f, v);
      }
    } else {
      // 8 rows of 64 at a time
#pragma nounroll
      for (int r = lane >> 3; r < 32; r += 8) {
        const lds_char *at = turn + r * TURN_ROW + (lane & 7) * 32;
        const f4 v[2] = {*(const lds_f4 *)at, *(const lds_f4 *)(at + 16)};
        if (EPI == EPI_ACT_GRAD) finish_gradient<T>(c, m1 + r, n0 + wn + (lane & 7) * 8, v);
        else finish_plain<T>(c, m1 + r, n0 + wn + (lane & 7) * 8, v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
#endif
}

template <class T, int A_KIND, int B_KIND, int DUAL, int EPI>
bool launch_product(int tile, const GemmCall &c, hipStream_t st) {
  const dim3 grid((uint32_t)(c.tiles_m * c.tiles_n), (uint32_t)(c.splits > 1 ? c.splits : 1));
  if (tile == TILE_256) hipLaunchKernelGGL((k_gemm<T, A_KIND, B_KIND, DUAL, EPI, 2, 4, 8>), grid, dim3(512), 0, st, c);
  else hipLaunchKernelGGL((k_gemm<T, A_KIND, B_KIND, DUAL, EPI, 2, 2, 4>), grid, dim3(256), 0, st, c);
  return hipGetLastError() == hipSuccess;
}

template <class T>
bool launch(int product, int tile, const GemmCall &c, void *stream) {
  hipStream_t st = (hipStream_t)stream;
  switch (product) {
    case GEMM_GATE_UP: return launch_product<T, ROWS, ROWS, 1, EPI_ACT>(tile, c, st);
    case GEMM_OUT: return launch_product<T, ROWS, ROWS, 0, EPI_STORE>(tile, c, st);
    case GEMM_DH: return launch_product<T, ROWS, COLS, 0, EPI_ACT_GRAD>(tile, c, st);
    case GEMM_DX: return launch_product<T, ROWS, COLS, 0, EPI_STORE>(tile, c, st);
    default: return launch_product<T, COLS, COLS, 0, EPI_STORE>(tile, c, st);
  }
}

}  // namespace chm_gemm
#endif

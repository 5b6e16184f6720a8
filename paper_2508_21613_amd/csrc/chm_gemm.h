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
// m.  Which rows of the tile a lane's n stand for is free; they are dealt out such that a lane ends with 16 consecutive n
// (8 features of the gate and of the up projection each in the two-weight product), which are stored as whole 16-byte words.
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

template <int N_SIDE, int DUAL> __device__ __forceinline__ uint32_t swz_rows(uint32_t row) {
  if (!N_SIDE) return row & 7u;
  if (DUAL) return (row & 3u) | (((row >> 3) & 1u) << 2);
  return (row & 3u) | (((row >> 4) & 1u) << 2);
}
template <int N_SIDE> __device__ __forceinline__ uint32_t swz_cols(uint32_t k) {
  if (!N_SIDE) return ((k & 3u) << 1) | (((k >> 3) & 1u) << 3);
  return (k & 1u) | (((k >> 1) & 1u) << 3) | (((k >> 3) & 1u) << 2);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const char *p, int64_t bytes) {
  const uint32_t n = bytes <= 0 ? 0u : bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes;
  return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)n, 0x00027000);
}

// One operand's way from memory to shared memory: W of its indices x BK sums a step, by NT threads.
template <int KIND, int N_SIDE, int DUAL, int W, int NT>
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
        const uint32_t row = idx / 8, chunk = (idx & 7u) ^ swz_rows<N_SIDE, DUAL>(row);
        const uint32_t r = DUAL ? (row >> 5) * 16 + (row & 15u) : row;
        off[i] = r * (uint32_t)ld_bytes + chunk * 16;
      } else {
        const uint32_t k = idx / (W / 8), chunk = (idx % (W / 8)) ^ swz_cols<N_SIDE>(k);
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
          const uint32_t row = (i * NT + tid) / 8, chunk = (tid & 7u) ^ swz_rows<N_SIDE, DUAL>(row);
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

// 8 sums of one index, from the tile in shared memory: `first` is the wavefront's first index, t its tile of 16
template <int KIND, int N_SIDE, int DUAL, int W>
__device__ __forceinline__ s8 fragment(const lds_char *lds, int first, int t, int ks, int lane) {
  const uint32_t q = lane >> 4, c = lane & 15;
  if (KIND == ROWS) {
    uint32_t row;
    if (!N_SIDE) row = first + t * 16 + c;
    else if (DUAL) row = first + (c >> 3) * 32 + (t >> 1) * 16 + ((c >> 2) & 1) * 8 + (t & 1) * 4 + (c & 3);
    else row = first + (c >> 2) * 16 + t * 4 + (c & 3);
    const uint32_t chunk = (ks * 4 + q) ^ swz_rows<N_SIDE, DUAL>(row);
    return *(const __attribute__((address_space(3))) s8 *)(lds + row * (BK * 2) + chunk * 16);
  }
  s4 half[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t k = ks * 32 + q * 8 + h * 4 + (c >> 2);
    uint32_t chunk, byte;
    if (!N_SIDE) { chunk = first / 8 + t * 2 + ((c & 3) >> 1); byte = (c & 1) * 8; }
    else { chunk = first / 8 + (c & 3) * 2 + (t >> 1); byte = (t & 1) * 8; }
    half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s4 *)(lds + k * (W * 2) + (chunk ^ swz_cols<N_SIDE>(k)) * 16 + byte));
  }
  return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
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

// stores `count` (<= N) of N consecutive values of one row
template <class T, int N>
__device__ __forceinline__ void store_row(const GemmCall &c, void *base, int64_t at, const float *v, int count) {
  if (c.f32_out) {
    float *p = (float *)base + at;
    if (c.wide && count >= N) {
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        f4 w = {v[i], v[i + 1], v[i + 2], v[i + 3]};
        if (c.accumulate) w += *(const f4 *)(p + i);
        *(f4 *)(p + i) = w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < count) p[i] = v[i] + (c.accumulate ? p[i] : 0.f);
    }
    return;
  }
  uint16_t *p = (uint16_t *)base + at;
  if (c.wide && count >= N) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      float w[8];
      const s8 old = c.accumulate ? *(const s8 *)(p + i) : s8{};
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = c.accumulate ? v[i + e] + T::up((uint16_t)old[e]) : v[i + e];
      *(s8 *)(p + i) = pack8<T>(w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < count) p[i] = T::down(c.accumulate ? v[i] + T::up(p[i]) : v[i]);
  }
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
  typedef Feed<A_KIND, 0, 0, TM, NT> FeedA;
  typedef Feed<B_KIND, 1, DUAL, TN, NT> FeedB;
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
  if (step < last) fetch(step, 0);
  int buf = 0;
  for (; step < last; ++step, buf ^= 1) {
    __syncthreads();                        // this step's tiles have arrived, the other buffer is read no more
    if (step + 1 < last) fetch(step + 1, buf ^ 1);
    const lds_char *ta = lds + buf * (FeedA::BYTES + FeedB::BYTES), *tb = ta + FeedA::BYTES;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      s8 b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = fragment<B_KIND, 1, DUAL, TN>(tb, wn, j, ks, lane);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const s8 a = fragment<A_KIND, 0, 0, TM>(ta, wm, t, ks, lane);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j][t] = T::mfma(b[j], a, acc[j][t]);
      }
    }
  }

  const int q = lane >> 4, r = lane & 15;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t m = m0 + wm + t * 16 + r;
    if (m >= c.m) continue;
    if (EPI == EPI_ACT) {
      // 8 features of both projections; the projections are rounded to 16 bits where they are kept for the backward pass,
      // their product is worked out from the float32 sums
      const int64_t f = n0 + wn / 2 + q * 8;        // rows of h are whole words of 8: what lies beyond the features is zero
      if (f >= c.n) continue;
      float g[8], u[8], h[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = acc[e >> 2][t][e & 3];
        u[e] = acc[2 + (e >> 2)][t][e & 3];
        h[e] = act_of(c.act, g[e]) * u[e];
        if (f + e >= c.n) g[e] = u[e] = h[e] = 0.f;
      }
      *(s8 *)(c.h + m * c.ldi + f) = pack8<T>(h);
      if (c.gate) {
        *(s8 *)(c.gate + m * c.ldi + f) = pack8<T>(g);
        *(s8 *)(c.up + m * c.ldi + f) = pack8<T>(u);
      }
    } else {
      const int64_t n = n0 + wn + q * 16;
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = acc[e >> 2][t][e & 3];
      if (EPI == EPI_ACT_GRAD) {
#pragma unroll
        for (int p = 0; p < 16; p += 8) {
          if (n + p >= c.n) continue;
          const s8 gs = *(const s8 *)(c.gate + m * c.ldi + n + p), us = *(const s8 *)(c.up + m * c.ldi + n + p);
          float h[8], dg[8], du[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float g = T::up((uint16_t)gs[e]), u = T::up((uint16_t)us[e]);
            float a, da;
            act_grad_of(c.act, g, a, da);
            h[e] = a * u;
            du[e] = v[p + e] * a;
            dg[e] = v[p + e] * u * da;
            if (n + p + e >= c.n_real) h[e] = du[e] = dg[e] = 0.f;
          }
          *(s8 *)(c.h + m * c.ldi + n + p) = pack8<T>(h);
          *(s8 *)(c.dgate + m * c.ldd + n + p) = pack8<T>(dg);
          *(s8 *)(c.dup + m * c.ldd + n + p) = pack8<T>(du);
        }
      } else if (c.splits > 1) {
        float *p = c.part + ((int64_t)blockIdx.y * c.m + m) * c.ld_part + n;
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          if (n + e < c.ld_part) *(f4 *)(p + e) = f4{v[e], v[e + 1], v[e + 2], v[e + 3]};
      } else {
        const int which = m >= c.m_first;
        const int64_t row = m - (which ? c.m_first : 0);
        if (row >= c.m_real || n >= c.n_real) continue;
        store_row<T, 16>(c, c.c[which], row * c.ldc + n, v, c.n_real - n < 16 ? (int)(c.n_real - n) : 16);
      }
    }
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

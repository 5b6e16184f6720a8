// Attention on the matrix cores: forward, the same for few rows, dq, and dk with dv.
//
//   z = cap tanh(scale q.k / cap) or scale q.k;  s = z - slope |i - j|;  p = exp(s - lse);  y = sum p v
//   ds = p (dy.v - delta) dz;  dq = scale sum ds k;  dk = scale sum ds q;  dv = sum p dy;  delta = dy.y
//
// Scores never leave the registers.  The products are taken so that a product's result is laid out as the next one's operand: in 32 x 32 x 16
// instructions a lane holds one column and, of its 32 rows, 4 h .. 4 h + 3 of every 8 (h: half of the wavefront).  With the keys as rows and the
// queries as columns a lane has one query (its maximum and sum need one exchange between the halves), and its 8 weights of 16 keys are the second
// operand of the next product, in whose first operand (values, transposed on their way from shared memory) the sums' order is the same.  dk and dv sum
// over queries: there the keys are the columns.
//
// Keys and values (queries and dy for dk and dv) go to shared memory by direct loads, 64 rows at a time, two such steps deep; 16-byte chunks
// of a row are stored at chunk ^ swizzle(row), which spreads both the reads of rows and the transposing reads over the banks.
//
// Tiles that nobody sees are not visited: each lane looks at one tile of 64 keys (of documents: least and largest number, prefix or not), and the
// ballot is the list of those to visit, and of those whose every pair is seen, where nothing is masked.
#ifndef CHM_ATTENTION_KERNELS_H
#define CHM_ATTENTION_KERNELS_H
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "chm_attention.h"

namespace chm_attention_kernels {

typedef float f16 __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

struct Bf16 {
  static __device__ __forceinline__ f16 mfma(s8 a, s8 b, f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
  static __device__ __forceinline__ float up(uint16_t u) { return __builtin_bit_cast(float, (uint32_t)u << 16); }
};
struct F16 {
  static __device__ __forceinline__ f16 mfma(s8 a, s8 b, f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
  static __device__ __forceinline__ float up(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
};

constexpr float LOWEST = -1.5e38f;          // reference of a row that has met nothing: finite, so that no difference of infinities arises
constexpr uint32_t OUT = 0x7fffffff;        // offset behind every buffer: reads as zero

__device__ __forceinline__ int divide(const AttnDivide &d, int n) { return d.m ? (int)(__umulhi((uint32_t)n, d.m) >> d.shift) : n; }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// the sum or maximum over both halves of the wavefront
__device__ __forceinline__ float both_max(float x) {
  const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float x) {
  const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <class T> __device__ __forceinline__ s8 pack8(const f16 &v, int from) {
  s8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (short)T::down(v[from + i]);
  return r;
}
// row of a 32 x 32 result in register r, less 4 h
__device__ __forceinline__ constexpr int row_of(int r) { return (r & 3) + 8 * (r >> 2); }

// ---------------------------------------------------------------------------------------------- shared memory
// Rows of D elements (64, or up to 128 in rows of 128).  Rows read: 16 lanes, 16 rows, one chunk each.  Transposing reads: 16 lanes, 4 rows,
// 2 chunks of each; the two halves of the wavefront 4 rows apart.  With 8 chunks a row, two rows fill the banks.
template <int D> struct Shape {
  enum { PITCH = D == 64 ? 128 : 256, CHUNKS = PITCH / 16, STEPS = D / 16, BLOCKS = D / 32 };
  static __device__ __forceinline__ uint32_t swizzle(uint32_t row) {
    return PITCH == 128 ? (row & 6u) | ((row >> 3) & 1u) : ((row & 7u) << 1) | ((row >> 3) & 1u);
  }
};

__device__ __forceinline__ i4 descriptor(const void *p, uint32_t bytes) {
  const uint64_t at = (uint64_t)p;
  i4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)at);
  r[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32) & 0xffff);
  r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
  r[3] = 0x00027000;
  return r;
}
// Written out, because the compiler otherwise waits for all loads under way before every transposing read of shared memory.  They write no register;
// the waits for what they bring are in arrived().
__device__ __forceinline__ void load_lds16(i4 rsrc, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(lds)));
}
__device__ __forceinline__ void load_lds4(i4 rsrc, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(lds)));
}
template <int PENDING> __device__ __forceinline__ void waited() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PENDING) : "memory"); }
// all loads under way and all reads of shared memory are back, then for the workgroup
__device__ __forceinline__ void arrived() {
  waited<0>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ROWS rows of keys or values to shared memory by NT threads; rows from `size` on and chunks from dim on arrive as zeros
template <int D, int ROWS, int NT>
struct KeyFeed {
  typedef Shape<D> S;
  enum { BYTES = ROWS * S::PITCH, LOADS = BYTES / 16 / NT };
  const char *base;
  int64_t token;                           // bytes from one to the next
  int32_t size, dim;
  uint32_t off[LOADS];
  __device__ __forceinline__ void start(const AttnInput &in, int b, int h, int size_, int dim_, int tid) {
    base = (const char *)(in.p + b * in.batch + h * in.head);
    token = in.token * 2;
    size = size_;
    dim = dim_;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t idx = i * NT + tid, row = idx / S::CHUNKS, chunk = (idx % S::CHUNKS) ^ S::swizzle(row);
      off[i] = (int)chunk * 8 >= dim ? OUT : row * (uint32_t)token + chunk * 16;
    }
  }
  // first: the first row (uniform)
  __device__ __forceinline__ void load(int first, uint32_t lds, int wave) const {
    const int left = size - first < ROWS ? size - first : ROWS;
    const i4 rsrc = descriptor(base + first * token, left > 0 ? (uint32_t)((left - 1) * (int32_t)token + dim * 2) : 0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_lds16(rsrc, off[i], lds + (i * NT + wave * 64) * 16);
  }
};

// ROWS rows of queries or dy
template <int D, int ROWS, int NT>
struct RowFeed {
  typedef Shape<D> S;
  enum { BYTES = ROWS * S::PITCH, LOADS = BYTES / 16 / NT };
  const char *base;
  int64_t token;
  uint32_t head;
  __device__ __forceinline__ void start(const AttnInput &in, int b, int first_head) {
    base = (const char *)(in.p + b * in.batch + first_head * in.head);
    token = in.token * 2;
    head = (uint32_t)in.head * 2;
  }
  __device__ __forceinline__ void load(const AttnCall &c, int first, uint32_t lds, int wave, int tid) const {
    const int t0 = divide(c.by_group, first);
    const i4 rsrc = descriptor(base + t0 * token, OUT - 64);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t idx = i * NT + tid, row = idx / S::CHUNKS, chunk = (idx % S::CHUNKS) ^ S::swizzle(row);
      const int r = first + (int)row, t = divide(c.by_group, r), g = r - t * c.group;
      const uint32_t off = (uint32_t)(t - t0) * (uint32_t)token + (uint32_t)g * head + chunk * 16;
      load_lds16(rsrc, r >= c.rows || (int)chunk * 8 >= c.dim ? OUT : off, lds + (i * NT + wave * 64) * 16);
    }
  }
};

// 8 elements (16 k + 8 h ..) of row `first` + lane % 32: operand of a product over a row's elements
template <int D>
__device__ __forceinline__ s8 row_fragment(const lds_char *lds, int first, int k, int lane) {
  const uint32_t row = first + (lane & 31), chunk = (k * 2 + (lane >> 5)) ^ Shape<D>::swizzle(row);
  return *(const __attribute__((address_space(3))) s8 *)(lds + row * Shape<D>::PITCH + chunk * 16);
}
// element 32 d + lane % 32 of the rows `first` + 4 h .. + 3 and 8 more on: operand of a product over rows
template <int D>
__device__ __forceinline__ s8 column_fragment(const lds_char *lds, int first, int d, int lane) {
  const uint32_t c = lane & 15;
  s4 half[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t row = first + (lane >> 5) * 4 + (c >> 2) + i * 8;
    const uint32_t chunk = (d * 4 + ((lane >> 4) & 1) * 2 + ((c & 3) >> 1)) ^ Shape<D>::swizzle(row);
    half[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(lds + row * Shape<D>::PITCH + chunk * 16 + (c & 1) * 8));
  }
  return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// rows of tokens that belong to no document may hold anything: zeros take their place where a product sums over them
template <int D, int ROWS, int NT>
__device__ __forceinline__ void clear_none(lds_char *lds, const uint32_t *words, int tid) {
  typedef Shape<D> S;
  for (int idx = tid; idx < ROWS * S::CHUNKS; idx += NT)
    if (words[idx / S::CHUNKS] == ATTN_NONE) *(__attribute__((address_space(3))) u4 *)(lds + idx * 16) = u4{0, 0, 0, 0};
}

// ---------------------------------------------------------------------------------------------- what is seen
struct Range { int first, last, flags; };   // documents of some tokens, as those of a tile

__device__ __forceinline__ Range join(Range a, const AttnTile &t) {
  return Range{t.first < a.first ? t.first : a.first, t.last > a.last ? t.last : a.last, a.flags | (t.flags & ATTN_SOME_NONE)};
}
// documents of the tokens [from, to] of a sequence, whole tiles of 64 of them
__device__ __forceinline__ Range range_of(const AttnTile *tiles, int from, int to) {
  Range r{INT32_MAX, -1, 0};
  for (int t = from / ATTN_TILE; t <= to / ATTN_TILE; ++t) r = join(r, tiles[t]);
  return r;
}

// whether queries at positions [from, to] of the documents `q` see some (all) of the keys [k0, k1]
__device__ __forceinline__ void sees(const AttnCall &c, int from, int to, const Range &q, int k0, int k1, const Range &k, bool &some, bool &all) {
  some = !c.causal || k0 <= to;
  all = !c.causal || k1 <= from;
  if (c.k_words) {
    some = (some || (k.flags & ATTN_SOME_PREFIX)) && k.first <= q.last && q.first <= k.last;
    all = (all || (k.flags & ATTN_ALL_PREFIX)) && !((k.flags | q.flags) & ATTN_SOME_NONE) && k.first == k.last && q.first == q.last && k.first == q.first;
  }
}

// Tiles of 64 keys that some rows see, in order: one that the workgroup visits, whether this wavefront does, whether it has to mask
struct KeyWalk {
  const AttnTile *tiles;
  int group_from, group_to, wave_from, wave_to;           // positions of the queries
  Range group_docs, wave_docs;
  int first, step;                          // every step-th tile from the first on: so the parts of split sums see equally much of any mask
  int at, end;                              // those of the present ballot: at .. at + 63; end: behind the last tile
  uint64_t visit, mine, mask, none;
  int tile;                                 // the present one; -1: no more
  bool run, masked, some_none;

  __device__ __forceinline__ void start(const AttnCall &c, int b, int group_row, int group_rows, int wave_row, int wave_rows, int first_, int step_, int end_) {
    tiles = c.k_words ? c.k_tiles + (int64_t)b * c.tiles : nullptr;
    const auto token = [&](int r) { return divide(c.by_group, r < c.rows ? r : c.rows - 1); };
    const int gf = token(group_row), gt = token(group_row + group_rows - 1), wf = token(wave_row), wt = token(wave_row + wave_rows - 1);
    group_from = gf + c.offset; group_to = gt + c.offset;
    wave_from = wf + c.offset; wave_to = wt + c.offset;
    if (tiles) {
      const AttnTile *q = c.q_tiles + (int64_t)b * c.q_tile_count;
      group_docs = range_of(q, gf, gt);
      wave_docs = range_of(q, wf, wt);
    }
    first = first_;
    step = step_;
    at = -64;
    end = end_;
    visit = 0;
  }
  __device__ __forceinline__ void next(const AttnCall &c, int lane) {
    while (!visit) {
      at += 64;
      if ((int64_t)at * step + first >= end) { tile = -1; return; }
      const int64_t tt = (int64_t)(at + lane) * step + first;
      const bool there = tt < end;
      const int t = there ? (int)tt : 0;
      Range k{0, 0, 0};
      if (tiles && there) { const AttnTile x = tiles[t]; k = Range{x.first, x.last, x.flags}; }
      const int k0 = t * ATTN_TILE, k1 = k0 + ATTN_TILE - 1;
      bool some, all, wave_some, wave_all;
      sees(c, group_from, group_to, group_docs, k0, k1, k, some, all);
      sees(c, wave_from, wave_to, wave_docs, k0, k1, k, wave_some, wave_all);
      visit = __ballot(there && some);
      mine = __ballot(there && wave_some);
      mask = __ballot(there && !(wave_all && k1 < c.keys));
      none = __ballot(there && tiles && (k.flags & ATTN_SOME_NONE));
    }
    const int i = __builtin_ctzll(visit);
    visit &= visit - 1;
    tile = (at + i) * step + first;
    run = (mine >> i) & 1;
    masked = (mask >> i) & 1;
    some_none = (none >> i) & 1;
  }
};

// Of the keys k0 + row_of(r): tells set(r, .) whether the query at `pos` of the document `word` sees it
template <class F>
__device__ __forceinline__ void seen_keys(const AttnCall &c, const uint32_t *words, int k0, int pos, uint32_t word, F set) {
  const int rel = words ? (c.causal ? pos - k0 : 64) : (c.causal && pos < c.keys - 1 ? pos : c.keys - 1) - k0;
  if (!words) {
#pragma unroll
    for (int r = 0; r < 16; ++r) set(r, row_of(r) <= rel);
    return;
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const u4 w = *(const u4 *)(words + k0 + g * 8);
    if (c.prefix) {
#pragma unroll
      for (int e = 0; e < 4; ++e) set(g * 4 + e, (w[e] == (word | 1u)) | ((w[e] == word) & (g * 8 + e <= rel)));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) set(g * 4 + e, (w[e] == word) & (g * 8 + e <= rel));
    }
  }
}

// a query's document as the comparisons want it: one that equals no key's where it has none
__device__ __forceinline__ uint32_t query_word(uint32_t word) { return word == ATTN_NONE ? ATTN_NOBODY : word & ~1u; }

// ---------------------------------------------------------------------------------------------- scores
// The score in powers of two from the product q.k.  CAP: the tanh is 1 - 2 / (1 + exp(2 x)), off by 2^-23 of the cap, not of itself, which is what
// a weight heeds.  `share` is 1 / (1 + exp(2 x)): the tanh's derivative is 4 share (1 - share).
template <int CAP>
__device__ __forceinline__ float capped(const AttnCall &c, float product, float &share) {
  if (!CAP) return product * c.to2;
  share = __builtin_amdgcn_rcpf(1.f + exp2_(product * c.tanh2));
  return fmaf(share, -2.f * c.cap2, c.cap2);
}
__device__ __forceinline__ float biased(float s, float slope2, float rel, int r) { return fmaf(-slope2, fabsf(rel - (float)row_of(r)), s); }

template <class T, int D, int NQ>
struct QueryRows {
  s8 q[NQ][D / 16];
  int pos[NQ];
  uint32_t word[NQ];
  float slope2[NQ];
  int row[NQ], token[NQ], head[NQ];
  // rows first + 32 n + lane % 32; those behind the last take its place (they are not stored)
  __device__ __forceinline__ void start(const AttnCall &c, int b, int h, int first, int lane) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      row[n] = first + n * 32 + (lane & 31);
      const int r = row[n] < c.rows ? row[n] : c.rows - 1;
      token[n] = divide(c.by_group, r);
      head[n] = h * c.group + r - token[n] * c.group;
      pos[n] = token[n] + c.offset;
      word[n] = c.q_words ? query_word(c.q_words[(int64_t)b * c.q_tile_count * ATTN_TILE + token[n]]) : 0;
      slope2[n] = c.slopes ? c.slopes[head[n]] * 1.44269504088896341f : 0.f;
      operand(c, c.q, b, n, lane, q[n]);
    }
  }
  // this lane's elements of its row n of another tensor of the queries' shape
  __device__ __forceinline__ void operand(const AttnCall &c, const AttnInput &in, int b, int n, int lane, s8 *out) const {
    const uint16_t *p = in.p + b * in.batch + token[n] * in.token + head[n] * in.head;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int d = k * 16 + (lane >> 5) * 8;
      out[k] = d < c.dim ? *(const s8 *)(p + d) : s8{};
    }
  }
};

// four consecutive elements d.. of a row of the results
template <class T>
__device__ __forceinline__ void store4(uint16_t *p, int d, int width, float a, float b, float e, float f) {
  const float v[4] = {a, b, e, f};
  if (d + 4 <= width) {
    typedef uint32_t u2_anywhere __attribute__((ext_vector_type(2), aligned(2)));
    u2_anywhere w;
    w[0] = (uint32_t)T::down(a) | ((uint32_t)T::down(b) << 16);
    w[1] = (uint32_t)T::down(e) | ((uint32_t)T::down(f) << 16);
    *(u2_anywhere *)(p + d) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < width) p[d + i] = T::down(v[i]);
  }
}

// what rounding took from them
template <class T>
__device__ __forceinline__ void store4_low(uint16_t *p, int d, int width, float a, float b, float e, float f) {
  store4<T>(p, d, width, a - T::up(T::down(a)), b - T::up(T::down(b)), e - T::up(T::down(e)), f - T::up(T::down(f)));
}

// One softmax over blocks of keys: running reference (powers of two) and sum.  The reference follows the maximum only when that has grown by more than
// 2^8: until then weights are up to 256, which 16-bit floats hold as exactly as smaller ones, and nothing has to be rescaled.
template <class T, int D, int NQ, int CAP, int SLOPE, int KB>
struct Softmax {
  f16 o[D / 32][NQ];
  float top[NQ], sum[NQ];
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      top[n] = LOWEST;
      sum[n] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d][n] = f16{};
    }
  }
  // KB blocks of 32 keys from key k0 on
  __device__ __forceinline__ void step(const AttnCall &c, const QueryRows<T, D, NQ> &rows, const uint32_t *words, const lds_char *keys, const lds_char *values, int k0,
                                       bool masked, int lane) {
    f16 s[KB][NQ];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[b][n] = f16{};
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const s8 a = row_fragment<D>(keys, b * 32, k, lane);
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[b][n] = T::mfma(a, rows.q[n][k], s[b][n]);
      }
    }
    const int h4 = (lane >> 5) * 4;
    constexpr bool RAW = !CAP && !SLOPE;    // then scores stay products until the exponential, which scales them
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float rel = SLOPE ? (float)(rows.pos[n] - (k0 + b * 32 + h4)) : 0.f;
        if (!RAW) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float share, v = capped<CAP>(c, s[b][n][r], share);
            if (SLOPE) v = biased(v, rows.slope2[n], rel, r);
            s[b][n][r] = v;
          }
        }
        if (masked) seen_keys(c, words, k0 + b * 32 + h4, rows.pos[n], rows.word[n], [&](int r, bool see) { s[b][n][r] = see ? s[b][n][r] : -INFINITY; });
      }
    const float unit = RAW ? c.to2 : 1.f;
    float most[NQ];
    bool grown = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float m = s[0][n][0];
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, s[b][n][r]);
      most[n] = both_max(m) * unit;
      grown = grown || most[n] > top[n] + 8.f;
    }
    if (__any(grown)) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float to = fmaxf(top[n], most[n]), f = exp2_(top[n] - to);
        top[n] = to;
        sum[n] *= f;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d][n] *= f;
      }
    }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      s8 p[NQ][2];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[b][n][r] = exp2_(RAW ? fmaf(s[b][n][r], c.to2, -top[n]) : s[b][n][r] - top[n]);
          sum[n] += s[b][n][r];
        }
        p[n][0] = pack8<T>(s[b][n], 0);
        p[n][1] = pack8<T>(s[b][n], 8);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const s8 a = column_fragment<D>(values, b * 32 + k * 16, d, lane);
#pragma unroll
          for (int n = 0; n < NQ; ++n) o[d][n] = T::mfma(a, p[n][k], o[d][n]);
        }
    }
  }
};

// ---------------------------------------------------------------------------------------------- forward
// which rows, of which sequence and key head, a workgroup works on: heads_abreast heads side by side (one a die where there are 8), the last rows first,
// which see the most
struct Place { int b, h, hb, tile, split; };
__device__ __forceinline__ Place place_of(const AttnCall &c, int tiles, bool last_first) {
  const int per = c.heads_abreast * tiles * c.splits;
  int i = blockIdx.x;
  const int band = i / per;
  i -= band * per;
  Place p;
  p.hb = band * c.heads_abreast + i % c.heads_abreast;
  i /= c.heads_abreast;
  p.split = i % c.splits;
  p.tile = i / c.splits;
  if (last_first) p.tile = tiles - 1 - p.tile;
  p.b = p.hb / c.kv_heads;
  p.h = p.hb - p.b * c.kv_heads;
  return p;
}

template <class T, int D, int NQ, int CAP, int SLOPE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) k_forward(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int KB = 2, WAVES = 4, NT = 64 * WAVES;
  typedef KeyFeed<D, ATTN_TILE, NT> Feed;
  __shared__ __attribute__((aligned(1024))) char shared[4 * Feed::BYTES];
  lds_char *lds = (lds_char *)shared;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place p = place_of(c, c.row_tiles, true);
  const int row0 = p.tile * (WAVES * NQ * 32), wave_row = row0 + wave * NQ * 32;
  QueryRows<T, D, NQ> rows;
  rows.start(c, p.b, p.h, wave_row, lane);
  Feed kf, vf;
  kf.start(c.k, p.b, p.h, c.keys, c.dim, tid);
  vf.start(c.v, p.b, p.h, c.keys, c.dim, tid);
  const uint32_t *words = c.k_words ? c.k_words + (int64_t)p.b * c.tiles * ATTN_TILE : nullptr;
  KeyWalk walk;
  walk.start(c, p.b, row0, WAVES * NQ * 32, wave_row, NQ * 32, p.split, c.splits, c.tiles);
  Softmax<T, D, NQ, CAP, SLOPE, KB> soft;
  soft.start();

  int slot = 0;
  walk.next(c, lane);
  if (walk.tile >= 0) {
    kf.load(walk.tile * ATTN_TILE, lds0, wave);
    vf.load(walk.tile * ATTN_TILE, lds0 + Feed::BYTES, wave);
  }
  while (walk.tile >= 0) {
    const int tile = walk.tile;
    const bool run = walk.run, masked = walk.masked, some_none = walk.some_none;
    walk.next(c, lane);
    arrived();                              // this tile is there, and the other slot has been read by everybody
    lds_char *here = lds + slot * 2 * Feed::BYTES;
    if (some_none) {
      clear_none<D, ATTN_TILE, NT>(here + Feed::BYTES, words + tile * ATTN_TILE, tid);
      arrived();
    }
    slot ^= 1;
    if (walk.tile >= 0) {
      kf.load(walk.tile * ATTN_TILE, lds0 + slot * 2 * Feed::BYTES, wave);
      vf.load(walk.tile * ATTN_TILE, lds0 + slot * 2 * Feed::BYTES + Feed::BYTES, wave);
    }
    if (run) soft.step(c, rows, words, here, here + Feed::BYTES, tile * ATTN_TILE, masked, lane);
  }

#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float sum = both_sum(soft.sum[n]);
    if (rows.row[n] >= c.rows) continue;
    const int h4 = (lane >> 5) * 4;
    if (c.splits > 1) {
      const int64_t at = ((int64_t)p.split * c.batch * c.kv_heads + p.hb) * c.rows + rows.row[n];
      float *out = c.part + at * c.width4;
      if (lane < 32) {
        c.part2[at * 2] = soft.top[n];
        c.part2[at * 2 + 1] = sum;
      }
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (d * 32 + g * 8 + h4 < c.width4)
            *(f4 *)(out + d * 32 + g * 8 + h4) = f4{soft.o[d][n][g * 4], soft.o[d][n][g * 4 + 1], soft.o[d][n][g * 4 + 2], soft.o[d][n][g * 4 + 3]};
      continue;
    }
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    if (c.lse && lane < 32) c.lse[(int64_t)p.hb * c.rows_pad + rows.row[n]] = sum == 0.f ? INFINITY : soft.top[n] + __builtin_amdgcn_logf(sum);
    uint16_t *out = c.y.p + p.b * c.y.batch + rows.token[n] * c.y.token + rows.head[n] * c.y.head;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4<T>(out, d * 32 + g * 8 + h4, c.width, soft.o[d][n][g * 4] * f, soft.o[d][n][g * 4 + 1] * f, soft.o[d][n][g * 4 + 2] * f, soft.o[d][n][g * 4 + 3] * f);
    if (!c.low) continue;
    out = c.low + (((int64_t)p.b * c.tokens + rows.token[n]) * (c.kv_heads * c.group) + rows.head[n]) * c.width;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4_low<T>(out, d * 32 + g * 8 + h4, c.width, soft.o[d][n][g * 4] * f, soft.o[d][n][g * 4 + 1] * f, soft.o[d][n][g * 4 + 2] * f, soft.o[d][n][g * 4 + 3] * f);
  }
#endif
}

// Up to 32 rows (the heads of a group for a token or a few) over many keys: bound by reading the keys and values.  Each wavefront has all rows, its
// own keys and its own shared memory, 32 keys at a time, and waits for nobody; the wavefronts' parts are joined at the end.
template <class T, int D, int CAP, int SLOPE>
__global__ void __launch_bounds__(256) k_forward_few(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WAVES = 4;
  typedef KeyFeed<D, 32, 64> Feed;
  constexpr int OWN = 4 * Feed::BYTES;      // two steps of keys and values; behind the loop 32 rows of D sums
  __shared__ __attribute__((aligned(1024))) char shared[WAVES * OWN];
  __shared__ float tops[WAVES][32], sums[WAVES][32];
  lds_char *lds = (lds_char *)shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  lds_char *own = lds + wave * OWN;
  const uint32_t own0 = (uint32_t)(uintptr_t)own;
  const Place p = place_of(c, 1, false);
  QueryRows<T, D, 1> rows;
  rows.start(c, p.b, p.h, 0, lane);
  Feed kf, vf;
  kf.start(c.k, p.b, p.h, c.keys, c.dim, lane);
  vf.start(c.v, p.b, p.h, c.keys, c.dim, lane);
  const uint32_t *words = c.k_words ? c.k_words + (int64_t)p.b * c.tiles * ATTN_TILE : nullptr;
  KeyWalk walk;
  walk.start(c, p.b, 0, 32, 0, 32, p.split * WAVES + wave, c.splits * WAVES, c.tiles);
  Softmax<T, D, 1, CAP, SLOPE, 1> soft;
  soft.start();

  int slot = 0, half = 0;
  walk.next(c, lane);
  if (walk.tile >= 0) {
    kf.load(walk.tile * ATTN_TILE, own0, 0);
    vf.load(walk.tile * ATTN_TILE, own0 + Feed::BYTES, 0);
  }
  while (walk.tile >= 0) {
    const int tile = walk.tile, k0 = tile * ATTN_TILE + half * 32;
    const bool masked = walk.masked, some_none = walk.some_none;
    half ^= 1;
    if (half == 0 || k0 + 32 >= c.keys) {
      half = 0;
      walk.next(c, lane);
    }
    lds_char *here = own + slot * 2 * Feed::BYTES;
    slot ^= 1;
    if (walk.tile >= 0) {
      const int k = walk.tile * ATTN_TILE + half * 32;
      kf.load(k, own0 + slot * 2 * Feed::BYTES, 0);
      vf.load(k, own0 + slot * 2 * Feed::BYTES + Feed::BYTES, 0);
      waited<2 * Feed::LOADS>();
    } else {
      waited<0>();
    }
    if (some_none) {
      clear_none<D, 32, 64>(here + Feed::BYTES, words + k0, lane);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    soft.step(c, rows, words, here, here + Feed::BYTES, k0, masked, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the slot has been read: the next loads go there
  }

  constexpr int PITCH = D + 4;              // floats: 32 rows of it in a wavefront's own memory
  static_assert(32 * PITCH * 4 <= OWN, "the sums of a wavefront");
  const float total = both_sum(soft.sum[0]);
  const int h4 = (lane >> 5) * 4;
  if (lane < 32) {
    tops[wave][lane] = soft.top[0];
    sums[wave][lane] = total;
  }
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(__attribute__((address_space(3))) f4 *)(own + ((lane & 31) * PITCH + d * 32 + g * 8 + h4) * 4) =
          f4{soft.o[d][0][g * 4], soft.o[d][0][g * 4 + 1], soft.o[d][0][g * 4 + 2], soft.o[d][0][g * 4 + 3]};
  __syncthreads();
  const int live = c.rows < 32 ? c.rows : 32;
  for (int i = tid; i < live * (D / 4); i += 256) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    float top = tops[0][r];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w][r]);
    float sum = 0.f;
    f4 v = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = exp2_(tops[w][r] - top);
      sum += sums[w][r] * f;
      v += *(const __attribute__((address_space(3))) f4 *)(lds + w * OWN + (r * PITCH + d) * 4) * f;
    }
    if (c.splits > 1) {
      const int64_t at = ((int64_t)p.split * c.batch * c.kv_heads + p.hb) * c.rows + r;
      if (d == 0) {
        c.part2[at * 2] = top;
        c.part2[at * 2 + 1] = sum;
      }
      if (d < c.width4) *(f4 *)(c.part + at * c.width4 + d) = v;
      continue;
    }
    const int token = divide(c.by_group, r), head = p.h * c.group + r - token * c.group;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    if (c.lse && d == 0) c.lse[(int64_t)p.hb * c.rows_pad + r] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
    store4<T>(c.y.p + p.b * c.y.batch + token * c.y.token + head * c.y.head, d, c.width, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
    if (c.low)
      store4_low<T>(c.low + (((int64_t)p.b * c.tokens + token) * (c.kv_heads * c.group) + head) * c.width, d, c.width, v[0] * f, v[1] * f, v[2] * f, v[3] * f);
  }
#endif
}

// ---------------------------------------------------------------------------------------------- backward
// p and ds of a score from the products q.k and dy.v; bias: of the distance, in powers of two
template <int CAP>
__device__ __forceinline__ void gradient(const AttnCall &c, float &s, float &dp, float bias, float lse, float delta) {
  float share, v = capped<CAP>(c, s, share);
  s = exp2_(v - bias - lse);
  dp = s * (dp - delta);
  if (CAP) dp *= 4.f * (share - share * share);
}

template <class T, int D, int NQ, int CAP, int SLOPE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) k_dq(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int KB = 2, WAVES = 4, NT = 64 * WAVES;
  typedef KeyFeed<D, ATTN_TILE, NT> Feed;
  __shared__ __attribute__((aligned(1024))) char shared[4 * Feed::BYTES];
  lds_char *lds = (lds_char *)shared;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place p = place_of(c, c.row_tiles, true);
  const int row0 = p.tile * (WAVES * NQ * 32), wave_row = row0 + wave * NQ * 32;
  QueryRows<T, D, NQ> rows;
  rows.start(c, p.b, p.h, wave_row, lane);
  s8 dy[NQ][D / 16];
  float lse[NQ], delta[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    rows.operand(c, c.dy, p.b, n, lane, dy[n]);
    const int r = rows.row[n] < c.rows ? rows.row[n] : c.rows - 1;
    const AttnRows &block = c.row_data[(int64_t)p.hb * (c.rows_pad / 32) + r / 32];
    lse[n] = block.lse[r % 32];
    delta[n] = block.delta[r % 32];
  }
  Feed kf, vf;
  kf.start(c.k, p.b, p.h, c.keys, c.dim, tid);
  vf.start(c.v, p.b, p.h, c.keys, c.dim, tid);
  const uint32_t *words = c.k_words ? c.k_words + (int64_t)p.b * c.tiles * ATTN_TILE : nullptr;
  KeyWalk walk;
  walk.start(c, p.b, row0, WAVES * NQ * 32, wave_row, NQ * 32, 0, 1, c.tiles);
  f16 dq[D / 32][NQ];
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int n = 0; n < NQ; ++n) dq[d][n] = f16{};

  int slot = 0;
  const int h4 = (lane >> 5) * 4;
  walk.next(c, lane);
  if (walk.tile >= 0) {
    kf.load(walk.tile * ATTN_TILE, lds0, wave);
    vf.load(walk.tile * ATTN_TILE, lds0 + Feed::BYTES, wave);
  }
  while (walk.tile >= 0) {
    const int tile = walk.tile;
    const bool run = walk.run, masked = walk.masked, some_none = walk.some_none;
    walk.next(c, lane);
    arrived();
    lds_char *here = lds + slot * 2 * Feed::BYTES;
    if (some_none) {
      clear_none<D, ATTN_TILE, NT>(here, words + tile * ATTN_TILE, tid);
      arrived();
    }
    slot ^= 1;
    if (walk.tile >= 0) {
      kf.load(walk.tile * ATTN_TILE, lds0 + slot * 2 * Feed::BYTES, wave);
      vf.load(walk.tile * ATTN_TILE, lds0 + slot * 2 * Feed::BYTES + Feed::BYTES, wave);
    }
    if (!run) continue;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const int k0 = tile * ATTN_TILE + b * 32 + h4;
      f16 s[NQ], dp[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n] = dp[n] = f16{};
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const s8 a = row_fragment<D>(here, b * 32, k, lane), v = row_fragment<D>(here + Feed::BYTES, b * 32, k, lane);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          s[n] = T::mfma(a, rows.q[n][k], s[n]);
          dp[n] = T::mfma(v, dy[n][k], dp[n]);
        }
      }
      s8 ds[NQ][2];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float rel = SLOPE ? (float)(rows.pos[n] - k0) : 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float x = s[n][r], y = dp[n][r];
          gradient<CAP>(c, x, y, SLOPE ? rows.slope2[n] * fabsf(rel - (float)row_of(r)) : 0.f, lse[n], delta[n]);
          dp[n][r] = y;
        }
        if (masked) seen_keys(c, words, k0, rows.pos[n], rows.word[n], [&](int r, bool see) { dp[n][r] = see ? dp[n][r] : 0.f; });
        ds[n][0] = pack8<T>(dp[n], 0);
        ds[n][1] = pack8<T>(dp[n], 8);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const s8 a = column_fragment<D>(here, b * 32 + k * 16, d, lane);
#pragma unroll
          for (int n = 0; n < NQ; ++n) dq[d][n] = T::mfma(a, ds[n][k], dq[d][n]);
        }
    }
  }
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    if (rows.row[n] >= c.rows) continue;
    uint16_t *out = c.dq.p + p.b * c.dq.batch + rows.token[n] * c.dq.token + rows.head[n] * c.dq.head;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        store4<T>(out, d * 32 + g * 8 + h4, c.width, dq[d][n][g * 4] * c.scale, dq[d][n][g * 4 + 1] * c.scale, dq[d][n][g * 4 + 2] * c.scale,
                  dq[d][n][g * 4 + 3] * c.scale);
  }
#endif
}

// Blocks of 32 rows that see some of a workgroup's keys, as KeyWalk
struct RowWalk {
  int group_from, group_to, wave_from, wave_to;           // keys
  Range group_docs, wave_docs;
  const AttnTile *tiles;                    // of the queries' tokens
  int first, step, at, end;
  uint64_t visit, mine, mask, none;
  int tile;
  bool run, masked, some_none;
  __device__ __forceinline__ void start(const AttnCall &c, int b, int group_key, int group_keys, int wave_key, int wave_keys, int first_, int step_, int end_) {
    group_from = group_key;
    group_to = group_key + group_keys - 1 < c.keys ? group_key + group_keys - 1 : c.keys - 1;
    wave_from = wave_key < c.keys ? wave_key : c.keys - 1;
    wave_to = wave_key + wave_keys - 1 < c.keys ? wave_key + wave_keys - 1 : c.keys - 1;
    tiles = nullptr;
    if (c.k_words) {
      tiles = c.q_tiles + (int64_t)b * c.q_tile_count;
      const AttnTile *k = c.k_tiles + (int64_t)b * c.tiles;
      group_docs = keys_of(k, group_from, group_to);
      wave_docs = keys_of(k, wave_from, wave_to);
    }
    first = first_;
    step = step_;
    at = -64;
    end = end_;
    visit = 0;
  }
  static __device__ __forceinline__ Range keys_of(const AttnTile *tiles, int from, int to) {
    Range r{INT32_MAX, -1, ATTN_ALL_PREFIX};
    for (int t = from / ATTN_TILE; t <= to / ATTN_TILE; ++t) {
      const AttnTile x = tiles[t];
      const int all = r.flags & x.flags & ATTN_ALL_PREFIX;
      r = join(r, x);
      r.flags = (r.flags & ~ATTN_ALL_PREFIX) | all | (x.flags & ATTN_SOME_PREFIX);
    }
    return r;
  }
  __device__ __forceinline__ void next(const AttnCall &c, int lane) {
    while (!visit) {
      at += 64;
      if ((int64_t)at * step + first >= end) { tile = -1; return; }
      const int64_t tt = (int64_t)(at + lane) * step + first;
      const bool there = tt < end;
      const int r0 = there ? (int)tt * 32 : 0, r1 = r0 + 31 < c.rows ? r0 + 31 : c.rows - 1;
      const int t0 = divide(c.by_group, r0), t1 = divide(c.by_group, r1);
      Range q{0, 0, 0};
      if (tiles) q = range_of(tiles, t0, t1);
      const int from = t0 + c.offset, to = t1 + c.offset;
      bool some, all, wave_some, wave_all;
      sees(c, from, to, q, group_from, group_to, group_docs, some, all);
      sees(c, from, to, q, wave_from, wave_to, wave_docs, wave_some, wave_all);
      visit = __ballot(there && some);
      mine = __ballot(there && wave_some);
      mask = __ballot(there && !(wave_all && r0 + 32 <= c.rows));
      none = __ballot(there && tiles && (q.flags & ATTN_SOME_NONE));
    }
    const int i = __builtin_ctzll(visit);
    visit &= visit - 1;
    tile = (at + i) * step + first;
    run = (mine >> i) & 1;
    masked = (mask >> i) & 1;
    some_none = (none >> i) & 1;
  }
};

// A wavefront has 32 keys: their operands, and 2 x 32 x D sums, which with the scores fill half of a lane's registers (two wavefronts a SIMD) if the
// values stay in shared memory: they are read from there a block, as the queries and dy are.
template <class T, int D, int CAP, int SLOPE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) k_dkdv(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WAVES = 4, NT = 64 * WAVES, KEYS = WAVES * 32;
  typedef RowFeed<D, 32, NT> Feed;
  typedef KeyFeed<D, KEYS, NT> Values;
  typedef __attribute__((address_space(3))) const AttnRows lds_rows;
  constexpr int STAGE = 2 * Feed::BYTES + 1024;            // queries, dy and what is known of 32 rows
  static_assert(sizeof(AttnRows) <= 1024, "a wavefront brings it in one load");
  __shared__ __attribute__((aligned(1024))) char shared[2 * STAGE + Values::BYTES];
  lds_char *lds = (lds_char *)shared, *values = lds + 2 * STAGE;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place p = place_of(c, c.key_tiles, false);
  const int key0 = p.tile * KEYS, wave_key = key0 + wave * 32;
  const int h4 = (lane >> 5) * 4;
  // this lane's key
  const int key = wave_key + (lane & 31), there = key < c.keys ? key : c.keys - 1;
  const uint32_t word = c.k_words ? c.k_words[(int64_t)p.b * c.tiles * ATTN_TILE + there] : 0;
  s8 k[D / 16];
  {
    const uint16_t *kp = c.k.p + p.b * c.k.batch + there * c.k.token + p.h * c.k.head;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int d = i * 16 + (lane >> 5) * 8;
      k[i] = d < c.dim ? *(const s8 *)(kp + d) : s8{};
    }
    Values vf;
    vf.start(c.v, p.b, p.h, c.keys, c.dim, tid);
    vf.load(key0, lds0 + 2 * STAGE, wave);
  }
  Feed qf, df;
  qf.start(c.q, p.b, p.h * c.group);
  df.start(c.dy, p.b, p.h * c.group);
  const uint32_t *q_words = c.q_words ? c.q_words + (int64_t)p.b * c.q_tile_count * ATTN_TILE : nullptr;
  const AttnRows *row_data = c.row_data + (int64_t)p.hb * (c.rows_pad / 32);

  // without a prefix a causal mask leaves the rows from the first key's position on
  const int blocks = (c.rows + 31) / 32;
  int first = 0;
  if (c.causal && !c.prefix && key0 > c.offset) {
    const int64_t f = (int64_t)(key0 - c.offset) * c.group / 32;
    first = f < blocks ? (int)f : blocks;
  }
  RowWalk walk;
  walk.start(c, p.b, key0, KEYS, wave_key, 32, first + p.split, c.splits, blocks);
  f16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f16{};

  const auto load = [&](int tile, int slot) {
    const uint32_t at = lds0 + slot * STAGE;
    qf.load(c, tile * 32, at, wave, tid);
    df.load(c, tile * 32, at + Feed::BYTES, wave, tid);
    if (wave == 0) load_lds16(descriptor(row_data + tile, sizeof(AttnRows)), lane * 16, at + 2 * Feed::BYTES);
  };
  int slot = 0;
  walk.next(c, lane);
  if (walk.tile >= 0) load(walk.tile, 0);
  while (walk.tile >= 0) {
    const int tile = walk.tile;
    const bool run = walk.run, masked = walk.masked, some_none = walk.some_none;
    walk.next(c, lane);
    arrived();
    lds_char *here = lds + slot * STAGE;
    if (some_none) {
      for (int idx = tid; idx < 32 * Shape<D>::CHUNKS; idx += NT) {
        const int r = tile * 32 + idx / Shape<D>::CHUNKS;
        if (r < c.rows && q_words[divide(c.by_group, r)] == ATTN_NONE) {
          *(__attribute__((address_space(3))) u4 *)(here + idx * 16) = u4{0, 0, 0, 0};
          *(__attribute__((address_space(3))) u4 *)(here + Feed::BYTES + idx * 16) = u4{0, 0, 0, 0};
        }
      }
      arrived();
    }
    slot ^= 1;
    if (walk.tile >= 0) load(walk.tile, slot);
    if (!run) continue;
    const lds_char *queries = here, *dys = here + Feed::BYTES;
    lds_rows *known = (lds_rows *)(here + 2 * Feed::BYTES);
    f16 s = {}, dp = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = T::mfma(row_fragment<D>(queries, 0, i, lane), k[i], s);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) dp = T::mfma(row_fragment<D>(dys, 0, i, lane), row_fragment<D>(values, wave * 32, i, lane), dp);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int r0 = g * 8 + h4;
      const f4 lse = *(__attribute__((address_space(3))) const f4 *)&known->lse[r0], delta = *(__attribute__((address_space(3))) const f4 *)&known->delta[r0];
      f4 bias = f4{0.f, 0.f, 0.f, 0.f};
      if (SLOPE) {
        const f4 slope2 = *(__attribute__((address_space(3))) const f4 *)&known->slope2[r0];
        const i4 pos = *(__attribute__((address_space(3))) const i4 *)&known->pos[r0];
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = slope2[e] * fabsf((float)(pos[e] - key));
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = s[g * 4 + e], y = dp[g * 4 + e];
        gradient<CAP>(c, x, y, bias[e], lse[e], delta[e]);
        s[g * 4 + e] = x;
        dp[g * 4 + e] = y;
      }
    }
    if (masked) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const i4 last = *(__attribute__((address_space(3))) const i4 *)&known->last[g * 8 + h4];
        const u4 words = *(__attribute__((address_space(3))) const u4 *)&known->word[g * 8 + h4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool before = key <= last[e], see = q_words ? (word == (words[e] | 1u)) | ((word == words[e]) & before) : before;
          s[g * 4 + e] = see ? s[g * 4 + e] : 0.f;
          dp[g * 4 + e] = see ? dp[g * 4 + e] : 0.f;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const s8 w = pack8<T>(s, i * 8), ds = pack8<T>(dp, i * 8);
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        dv[d] = T::mfma(column_fragment<D>(dys, i * 16, d, lane), w, dv[d]);
        dk[d] = T::mfma(column_fragment<D>(queries, i * 16, d, lane), ds, dk[d]);
      }
    }
  }
  if (walk.tile < 0) waited<0>();           // the values, where no block was visited
  if (key >= c.keys) return;
  if (c.splits > 1) {
    const int64_t at = (((int64_t)p.split * c.batch * c.kv_heads + p.hb) * c.keys + key) * c.width4;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int e = d * 32 + g * 8 + h4;
        if (e >= c.width4) continue;
        *(f4 *)(c.part + at + e) = f4{dk[d][g * 4], dk[d][g * 4 + 1], dk[d][g * 4 + 2], dk[d][g * 4 + 3]} * c.scale;
        *(f4 *)(c.part2 + at + e) = f4{dv[d][g * 4], dv[d][g * 4 + 1], dv[d][g * 4 + 2], dv[d][g * 4 + 3]};
      }
    return;
  }
  uint16_t *ko = c.dk.p + p.b * c.dk.batch + key * c.dk.token + p.h * c.dk.head, *vo = c.dv.p + p.b * c.dv.batch + key * c.dv.token + p.h * c.dv.head;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      store4<T>(ko, d * 32 + g * 8 + h4, c.width, dk[d][g * 4] * c.scale, dk[d][g * 4 + 1] * c.scale, dk[d][g * 4 + 2] * c.scale, dk[d][g * 4 + 3] * c.scale);
      store4<T>(vo, d * 32 + g * 8 + h4, c.width, dv[d][g * 4], dv[d][g * 4 + 1], dv[d][g * 4 + 2], dv[d][g * 4 + 3]);
    }
#endif
}

// ---------------------------------------------------------------------------------------------- launches
enum { FORWARD, FEW, DQ, DKDV };
template <class T, int WHAT, int D, int N, int CAP, int SLOPE>
bool launch(const AttnCall &c, const AttnLaunch &l) {
  hipStream_t st = (hipStream_t)l.stream;
  const dim3 grid(l.groups), block(256);
  if constexpr (WHAT == FORWARD) hipLaunchKernelGGL((k_forward<T, D, N, CAP, SLOPE>), grid, block, 0, st, c);
  else if constexpr (WHAT == FEW) hipLaunchKernelGGL((k_forward_few<T, D, CAP, SLOPE>), grid, block, 0, st, c);
  else if constexpr (WHAT == DQ) hipLaunchKernelGGL((k_dq<T, D, N, CAP, SLOPE>), grid, block, 0, st, c);
  else hipLaunchKernelGGL((k_dkdv<T, D, CAP, SLOPE>), grid, block, 0, st, c);
  return hipGetLastError() == hipSuccess;
}
template <class T, int WHAT, int D, int N>
bool launch_terms(const AttnCall &c, const AttnLaunch &l) {
  const bool cap = c.cap2 != 0.f, slope = c.slopes != nullptr;
  if (cap) return slope ? launch<T, WHAT, D, N, 1, 1>(c, l) : launch<T, WHAT, D, N, 1, 0>(c, l);
  return slope ? launch<T, WHAT, D, N, 0, 1>(c, l) : launch<T, WHAT, D, N, 0, 0>(c, l);
}
template <class T, int WHAT>
bool launch_shape(const AttnCall &c, const AttnLaunch &l) {
  return l.dim == 64 ? launch_terms<T, WHAT, 64, 1>(c, l) : launch_terms<T, WHAT, 128, 1>(c, l);
}

}  // namespace chm_attention_kernels
#endif

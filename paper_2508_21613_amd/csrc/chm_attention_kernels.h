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
// Keys and values (queries and dy for dk and dv) go to shared memory by direct loads, 64 (32) rows at a time, two such steps deep; 16-byte chunks
// of a row are stored at chunk ^ swizzle(row), which spreads both the reads of rows and the transposing reads over the banks.
//
// Two wavefronts a SIMD, each of whose steps is 1,024 cycles of matrix instructions, as many of other ones and 32 KB (forward) from shared memory.  In long calls little
// of one's work runs beside the other's: matrix core and vector unit are busy for 39 and 66% of the time in the forward pass, 44 and 60% in dq, 42 and 46% in dk and dv (shared memory 20 to 32%), without
// a cap for 50 and 47, 59 and 41, 49 and 29%, at 1.8 to 2.1 GHz of 2.4.  8,192 tokens, 32 heads of 128, 8 of keys, bfloat16, causal, capped, call after call: forward
// 650 us (0.85 PFLOP/s of the 4 d operations a pair), dq 885 (0.93 of 6 d), dk and dv 1,225 (0.90 of 8 d); without the cap 547, 735, 1,058 (1.00, 1.12, 1.04).  The first calls
// after a pause take up to a fifth longer.
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
typedef __attribute__((address_space(3))) const uint32_t lds_word;

// LIFT: the gradients' p and ds are worked out 2^LIFT times as large, and their sums taken down again at the end.  Bf16 reaches as far down as float32; float16's
// least step, 2^-24, is much of a ds of 1 / keys and a small dy long before the results come near it (4,096 keys, 128 elements, no mask: dk off by 8.1e-4 with a dy
// of 1e-3 and by 3.4e-3 with one of 2e-4, with the lift by 3.0e-4 and 3.5e-4, where rounding it alone takes 2.1e-4 and 2.8e-4).  2^16 / 2^12 leaves p room for what rounding does to scores of up to 2^26; ds has lower().
struct Bf16 {
  enum { LIFT = 0 };
  static __device__ __forceinline__ f16 mfma(s8 a, s8 b, f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
  static __device__ __forceinline__ float up(uint16_t u) { return __builtin_bit_cast(float, (uint32_t)u << 16); }
};
struct F16 {
  enum { LIFT = 12 };
  static __device__ __forceinline__ f16 mfma(s8 a, s8 b, f16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint16_t down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
  static __device__ __forceinline__ float up(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
};

constexpr float LOWEST = -1.5e38f;          // reference of a row that has met nothing: finite, so that no difference of infinities arises
constexpr uint32_t OUT = 0x7fffffff;        // offset behind every buffer: reads as zero

__device__ __forceinline__ int divide(const AttnDivide &d, int n) { return d.m ? (int)(__umulhi((uint32_t)n, d.m) >> d.shift) : n; }
// the lane's number, worked out where it is used and nowhere before: for loops that have no register left
__device__ __forceinline__ int own_lane() {
  int lane;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(lane));
  return lane;
}
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
// what pack8 takes from them
template <class T> __device__ __forceinline__ s8 pack8_low(const f16 &v, const s8 &high, int from) {
  s8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (short)T::down(v[from + i] - T::up((uint16_t)high[i]));
  return r;
}
// row of a 32 x 32 result in register r, less 4 h
__device__ __forceinline__ constexpr int row_of(int r) { return (r & 3) + 8 * (r >> 2); }

// The call's description as the kernel's argument holds it, read anew: what only the end of a kernel asks for is otherwise kept in scalar registers from
// its beginning, which then lack in its loop (dk and dv: 45 reads of saved ones a step).
typedef __attribute__((address_space(4))) const AttnCall Argument;
__device__ __forceinline__ Argument *argument() {
  Argument *c = (Argument *)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(c));
  return c;
}

// which rows, of which sequence and key head, a workgroup works on: heads_abreast heads side by side (one a die where there are 8), the last rows first,
// which see the most
struct Place { int b, h, hb, tile, split; };
__device__ __forceinline__ Place place_of(const AttnCall &c, int i, bool last_first) {
  Place p;
  const int j = divide(c.by_abreast, i), k = divide(c.by_splits, j), band = divide(c.by_tiles, k);
  p.split = j - k * c.splits;
  p.tile = k - band * c.tiles_here;
  if (last_first) p.tile = c.tiles_here - 1 - p.tile;
  p.hb = band * c.heads_abreast + i - j * c.heads_abreast;
  p.b = divide(c.by_kv_heads, p.hb);
  p.h = p.hb - p.b * c.kv_heads;
  return p;
}

// ---------------------------------------------------------------------------------------------- shared memory
// Rows of D elements (64, or up to 128 in rows of 128), as direct loads leave them: 1 KiB of whole rows by each.  Laid out for 64 banks of 4 bytes: 16 lanes of
// a read of rows, one chunk of 16 rows each, or 32 lanes of a transposing read, 4 chunks of 4 rows, go to all of them once.  The chunks of a row are exchanged in fours by
// the row's last two bits, and 16 bytes between the loads do the rest: so most of a read's address is a constant.  With 8 chunks a row, where two rows
// fill the banks, they are exchanged by three bits of the row.  Measured in long calls: conflicts are 0.3 to 0.7% of shared memory's busy cycles.
template <int D> struct Shape {
  enum { PITCH = D == 64 ? 128 : 256, CHUNKS = PITCH / 16, GROUP = 1024 / PITCH, GROUP_BYTES = 1024 + (D == 64 ? 0 : 16) };
  static __device__ __forceinline__ uint32_t swizzle(uint32_t row) {
    return PITCH == 128 ? ((row & 2u) << 1) | ((row >> 2) & 3u) : (row & 3u) << 2;
  }
  static __device__ __forceinline__ constexpr uint32_t row_at(uint32_t row) { return row / GROUP * GROUP_BYTES + row % GROUP * PITCH; }
  static constexpr int bytes(int rows) { return rows / GROUP * GROUP_BYTES; }
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

// ROWS rows of keys or values to shared memory by WAVES wavefronts; rows from `size` on and chunks from dim on arrive as zeros.
template <int D, int ROWS, int WAVES>
struct KeyFeed {
  typedef Shape<D> S;
  enum { BYTES = S::bytes(ROWS), LOADS = ROWS / S::GROUP / WAVES };
  const char *base;
  int64_t token;                           // bytes from one to the next
  int32_t size, dim;
  uint32_t off[LOADS];
  __device__ __forceinline__ void start(const AttnInput &in, int b, int h, int size_, int dim_, int wave, int lane) {
    base = (const char *)(in.p + b * in.batch + h * in.head);
    token = in.token * 2;
    size = size_;
    dim = dim_;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint32_t idx = (i * WAVES + wave) * 64 + lane, row = idx / S::CHUNKS, chunk = (idx % S::CHUNKS) ^ S::swizzle(row);
      off[i] = (int)chunk * 8 >= dim ? OUT : row * (uint32_t)token + chunk * 16;
    }
  }
  // the rows from `first` on (uniform)
  __device__ __forceinline__ void load(int first, uint32_t lds, int wave) const {
    const int left = size - first < ROWS ? size - first : ROWS;
    const i4 rsrc = descriptor(base + first * token, left > 0 ? (uint32_t)((left - 1) * (int32_t)token + dim * 2) : 0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_lds16(rsrc, off[i], lds + (i * WAVES + wave) * S::GROUP_BYTES);
  }
};

// ROWS rows of queries or dy.  Where the group divides 32 every block of rows starts with a token, and a lane's offsets stay what they are; worked out
// anew for every block they cost a sixth of the time of dk and dv.
template <int D, int ROWS, int WAVES>
struct RowFeed {
  typedef Shape<D> S;
  enum { BYTES = S::bytes(ROWS), LOADS = ROWS / S::GROUP / WAVES };
  const char *base;
  int64_t token;
  uint32_t head, off[LOADS];
  __device__ __forceinline__ void start(const AttnInput &in, int b, int first_head) {
    base = (const char *)(in.p + b * in.batch + first_head * in.head);
    token = in.token * 2;
    head = (uint32_t)in.head * 2;
  }
  __device__ __forceinline__ void keep(const AttnCall &c, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) off[i] = offset(c, i, 0, 0, wave, lane);
  }
  __device__ __forceinline__ uint32_t offset(const AttnCall &c, int i, int first, int t0, int wave, int lane) const {
    const uint32_t idx = (i * WAVES + wave) * 64 + lane, row = idx / S::CHUNKS, chunk = (idx % S::CHUNKS) ^ S::swizzle(row);
    const int r = first + (int)row, t = divide(c.by_group, r), g = r - t * c.group;
    return r >= c.rows || (int)chunk * 8 >= c.dim ? OUT : (uint32_t)(t - t0) * (uint32_t)token + (uint32_t)g * head + chunk * 16;
  }
  // the rows from `first` on (uniform), which may lie behind the last
  __device__ __forceinline__ void once(const AttnCall &c, int first, uint32_t lds, int lane) const {
    const int t0 = divide(c.by_group, first < c.rows ? first : c.rows - 1);
    const i4 rsrc = descriptor(base + t0 * token, OUT - 64);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_lds16(rsrc, offset(c, i, first, t0, 0, lane), lds + i * S::GROUP_BYTES);
  }
  // the rows from `first` on, again and again
  __device__ __forceinline__ void load(const AttnCall &c, int first, uint32_t lds, int wave, int lane) const {
    const int t0 = divide(c.by_group, first);
    const i4 rsrc = descriptor(base + t0 * token, OUT - 64);
    if (c.even_group && first + ROWS <= c.rows) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_lds16(rsrc, off[i], lds + (i * WAVES + wave) * S::GROUP_BYTES);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) load_lds16(rsrc, offset(c, i, first, t0, wave, lane), lds + (i * WAVES + wave) * S::GROUP_BYTES);
    }
  }
};

// 8 elements (16 k + 8 h ..) of row `first` + lane % 32: operand of a product over a row's elements.  first: a multiple of 32
template <int D>
__device__ __forceinline__ s8 row_fragment(const lds_char *lds, int first, int k, int lane) {
  typedef Shape<D> S;
  const uint32_t row = lane & 31, chunk = (k * 2 + (lane >> 5)) ^ S::swizzle(row);
  return *(const __attribute__((address_space(3))) s8 *)(lds + S::row_at(first) + S::row_at(row) + chunk * 16);
}
// element 32 d + lane % 32 of the rows `first` + 4 h .. + 3 and 8 more on: operand of a product over rows.  first: a multiple of 16
template <int D>
__device__ __forceinline__ s8 column_fragment(const lds_char *lds, int first, int d, int lane) {
  typedef Shape<D> S;
  const uint32_t c = lane & 15, row = (lane >> 5) * 4 + (c >> 2);
  s4 half[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t chunk = (d * 4 + ((lane >> 4) & 1) * 2 + ((c & 3) >> 1)) ^ S::swizzle(row + i * 8);      // first changes none of the bits
    half[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(lds + S::row_at(first + i * 8) + S::row_at(row) + chunk * 16 + (c & 1) * 8));
  }
  return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// rows of tokens that belong to no document may hold anything: zeros take their place where a product sums over them
template <int D>
__device__ __forceinline__ void clear_row(lds_char *lds, int row, int chunk) {
  *(__attribute__((address_space(3))) u4 *)(lds + Shape<D>::row_at(row) + chunk * 16) = u4{0, 0, 0, 0};
}
template <int D, int ROWS, int NT>
__device__ __forceinline__ void clear_none(lds_char *lds, const uint32_t *words, int tid) {
  for (int idx = tid; idx < ROWS * Shape<D>::CHUNKS; idx += NT)
    if (words[idx / Shape<D>::CHUNKS] == ATTN_NONE) clear_row<D>(lds, idx / Shape<D>::CHUNKS, idx % Shape<D>::CHUNKS);
}

// A tile of 64 keys, their values and words, in one of two slots
template <int D, int WAVES>
struct TileFeed {
  typedef KeyFeed<D, ATTN_TILE, WAVES> Feed;
  enum { VALUES = Feed::BYTES, WORDS = 2 * Feed::BYTES, SLOT = WORDS + ATTN_TILE * 4, BYTES = 2 * SLOT };
  Feed keys, values;
  const uint32_t *words;                   // null: none
  __device__ __forceinline__ void start(const AttnCall &c, const Place &p, int wave, int lane) {
    keys.start(c.k, p.b, p.h, c.keys, c.dim, wave, lane);
    values.start(c.v, p.b, p.h, c.keys, c.dim, wave, lane);
    words = c.k_words ? c.k_words + (int64_t)p.b * c.tiles * ATTN_TILE : nullptr;
  }
  __device__ __forceinline__ void load(int tile, uint32_t lds, int wave, int lane) const {
    keys.load(tile * ATTN_TILE, lds, wave);
    values.load(tile * ATTN_TILE, lds + VALUES, wave);
    if (words && wave == 0) load_lds4(descriptor(words + (int64_t)tile * ATTN_TILE, ATTN_TILE * 4), lane * 4, lds + WORDS);
  }
  // zeros in the rows at `rows` of keys of no document
  __device__ __forceinline__ static void clear(lds_char *slot, lds_char *rows, int tid) {
    lds_word *w = (lds_word *)(slot + WORDS);
    for (int idx = tid; idx < ATTN_TILE * Shape<D>::CHUNKS; idx += 64 * WAVES)
      if (w[idx / Shape<D>::CHUNKS] == ATTN_NONE) clear_row<D>(rows, idx / Shape<D>::CHUNKS, idx % Shape<D>::CHUNKS);
  }
};

// ---------------------------------------------------------------------------------------------- what is seen
struct Range { int first, last, flags; };   // documents of some tokens, as those of a tile

__device__ __forceinline__ Range join(Range a, const AttnTile &t) {
  return Range{t.first < a.first ? t.first : a.first, t.last > a.last ? t.last : a.last, a.flags | (t.flags & ATTN_SOME_NONE)};
}
// documents of the tokens [from, to] of a sequence, whole tiles of 64 of them, of which there are at most N: all are asked for at once
template <int N>
__device__ __forceinline__ Range range_of(const AttnTile *tiles, int from, int to) {
  AttnTile x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = tiles[from / ATTN_TILE + i < to / ATTN_TILE ? from / ATTN_TILE + i : to / ATTN_TILE];
  Range r{INT32_MAX, -1, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) r = join(r, x[i]);
  return r;
}

// documents of the words of a wavefront's lanes, the same for all of it
__device__ __forceinline__ Range range_of(uint32_t word) {
  const uint32_t one = __builtin_amdgcn_readfirstlane(word);
  if (__all(word == one)) return one == ATTN_NONE ? Range{INT32_MAX, -1, ATTN_SOME_NONE} : Range{(int)(one >> 1), (int)(one >> 1), one & 1 ? ATTN_SOME_PREFIX | ATTN_ALL_PREFIX : 0};
  const bool none = word == ATTN_NONE;
  int lo = none ? INT32_MAX : (int)(word >> 1), hi = none ? -1 : (int)(word >> 1);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const int l = __shfl_xor(lo, d), h = __shfl_xor(hi, d);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
  }
  const uint64_t pre = __ballot(!none && (word & 1));
  return Range{__builtin_amdgcn_readfirstlane(lo), __builtin_amdgcn_readfirstlane(hi),
               (__any(none) ? ATTN_SOME_NONE : 0) | (pre ? ATTN_SOME_PREFIX : 0) | (pre == ~0ull ? ATTN_ALL_PREFIX : 0)};
}

// What queries at positions [from, to] of the documents `q` see of the keys [k0, k1]: some; all as far as documents go; all as far as their order goes
struct Sight { bool some, documents, order; };
__device__ __forceinline__ Sight sees(const AttnCall &c, int from, int to, const Range &q, int k0, int k1, const Range &k) {
  Sight s{!c.causal || k0 <= to, true, !c.causal || k1 <= from};
  if (c.k_words) {
    s.some = (s.some || (k.flags & ATTN_SOME_PREFIX)) && k.first <= q.last && q.first <= k.last;
    s.documents = !((k.flags | q.flags) & ATTN_SOME_NONE) && k.first == k.last && q.first == q.last && k.first == q.first;
    s.order = s.order || (k.flags & ATTN_ALL_PREFIX);
  }
  return s;
}

// A tile that the workgroup visits (-1: no more), whether this wavefront does, what it has to mask, whether there are places of no document.  Most
// tiles of packed documents lie within one, so that only their order is asked for, or the documents where one ends.
struct Visit {
  int tile;
  bool run, documents, order, some_none;
  __device__ __forceinline__ bool masked() const { return documents | order; }
};

// Tiles of 64 keys that some of ROWS rows see, in order; a wavefront has 32 of them
template <int ROWS>
struct KeyWalk {
  const AttnTile *tiles;
  int group_from, group_to, wave_from, wave_to;           // positions of the queries
  Range group_docs, wave_docs;             // the wavefront's are its own rows' (a tile of the queries may hold two documents)
  int first, step;                          // every step-th tile from the first on: so the parts of split sums see equally much of any mask
  int at, end;                              // those of the present ballot: at .. at + 63; end: behind the last tile
  uint64_t visit, mine, documents, order, none;

  // word: of the lane's row.  The first 64 tiles are asked for along with all else that is needed to choose among them.
  __device__ __forceinline__ void start(const AttnCall &c, int b, int group_row, int wave_row, uint32_t word, int first_, int step_, int end_, int lane) {
    tiles = c.k_words ? c.k_tiles + (int64_t)b * c.tiles : nullptr;
    const auto token = [&](int r) { return divide(c.by_group, r < c.rows ? r : c.rows - 1); };
    const int gf = token(group_row), gt = token(group_row + ROWS - 1), wf = token(wave_row), wt = token(wave_row + 31);
    group_from = gf + c.offset; group_to = gt + c.offset;
    wave_from = wf + c.offset; wave_to = wt + c.offset;
    first = first_;
    step = step_;
    at = 0;
    end = end_;
    const AttnTile x = documents_of(lane);
    if (tiles) {
      group_docs = range_of<ROWS / 64 + 1>(c.q_tiles + (int64_t)b * c.q_tile_count, gf, gt);
      wave_docs = range_of(word);
    }
    choose(c, x, lane);
  }
  // of the lane's tile of the present 64
  __device__ __forceinline__ AttnTile documents_of(int lane) const {
    const int64_t t = (int64_t)(at + lane) * step + first;
    return tiles && t < end ? tiles[t] : AttnTile{0, 0, 0, 0};
  }
  __device__ __forceinline__ void choose(const AttnCall &c, const AttnTile &x, int lane) {
    const int64_t tt = (int64_t)(at + lane) * step + first;
    const bool there = tt < end;
    const int t = there ? (int)tt : 0, k0 = t * ATTN_TILE, k1 = k0 + ATTN_TILE - 1;
    const Range k{x.first, x.last, x.flags};
    const Sight group = sees(c, group_from, group_to, group_docs, k0, k1, k), wave = sees(c, wave_from, wave_to, wave_docs, k0, k1, k);
    visit = __ballot(there && group.some);
    mine = __ballot(there && wave.some);
    documents = __ballot(there && tiles && !(wave.documents && k1 < c.keys));           // places behind the last key are of no document
    order = __ballot(there && !(wave.order && (tiles || k1 < c.keys)));
    none = __ballot(there && tiles && (k.flags & ATTN_SOME_NONE));
  }
  __device__ __forceinline__ Visit next(const AttnCall &c, int lane) {
    while (!visit) {
      if ((int64_t)(at + 64) * step + first >= end) return Visit{-1, false, false, false, false};
      at += 64;
      choose(c, documents_of(lane), lane);
    }
    const int i = __builtin_ctzll(visit);
    visit &= visit - 1;
    return Visit{(at + i) * step + first, (bool)((mine >> i) & 1), (bool)((documents >> i) & 1), (bool)((order >> i) & 1), (bool)((none >> i) & 1)};
  }
};

// Masks are 32 bits a lane, one for each key (row) of a block: worked out once, and each score costs two operations that wait for no comparison (4,096 packed
// tokens, 32 heads of 128, 8 of keys: forward 74 -> 71 us, dq 99 -> 94).  A bit of `there` (the
// lane's place in the block) whose word is the lane's own: a ballot for each document of the wavefront, of which there is mostly one.
__device__ __forceinline__ uint32_t same_words(uint32_t own, uint32_t there) {
  uint32_t bits = 0;
  uint64_t left = ~0ull;
  do {
    const uint32_t one = __builtin_amdgcn_readlane(own, __builtin_ctzll(left));
    const uint64_t lanes = __ballot(own == one);
    const uint32_t equal = (uint32_t)__ballot(there == one);
    bits = own == one ? equal : bits;
    left &= ~lanes;
  } while (left);
  return bits;
}
// Of the 32 keys from k0 on those that the query at `pos` of the document `word` sees, as far as `now` asks (the wavefront's other tiles need no mask); there:
// word of the key k0 + lane % 32.  Bit row_of(r): that of a score's register r
__device__ __forceinline__ uint32_t seen_keys(const AttnCall &c, const Visit &now, uint32_t there, int k0, int pos, uint32_t word, int lane) {
  uint32_t seen = now.documents ? same_words(word, there & ~1u) : ~0u;
  if (now.order) {
    const int rel = (c.causal && (c.k_words || pos < c.keys - 1) ? pos : c.keys - 1) - k0;
    uint32_t before = rel < 0 ? 0u : rel > 30 ? ~0u : (2u << rel) - 1;
    if (c.prefix) before |= (uint32_t)__ballot(there & 1);
    seen &= before;
  }
  return seen >> (lane >> 5) * 4;
}
// v where the bit of register r is set, `hidden` elsewhere
__device__ __forceinline__ float where_seen(uint32_t seen, int r, float v, uint32_t hidden) {
  const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)seen, row_of(r), 1);
  return __uint_as_float((__float_as_uint(v) & keep) | (hidden & ~keep));
}

// a query's document as the comparisons want it: one that equals no key's where it has none
__device__ __forceinline__ uint32_t query_word(uint32_t word) { return word == ATTN_NONE ? ATTN_NOBODY : word; }

// ---------------------------------------------------------------------------------------------- scores
// The score in powers of two from the product q.k, and `share` = 1 / (1 + exp(2 x)), x = score / cap: the tanh is 1 - 2 share, off by 2^-23 of the cap, not of
// itself, and its derivative 4 share (1 - share).  That is what weights heed as long as the cap is not large.  CAP = 2, for large ones: scores up to 1 / 4 of
// the cap are score (1 - x^2 / 3 + 2 x^4 / 15 - 17 x^6 / 315), where the next term is 2^-21 and less.
template <int CAP>
__device__ __forceinline__ float capped(const AttnCall &c, float product, float &share) {
  if (!CAP) return product * c.to2;
  share = __builtin_amdgcn_rcpf(1.f + exp2_(product * c.tanh2));
  const float far = fmaf(share, -2.f * c.cap2, c.cap2);
  if (CAP == 1) return far;
  const float x = product * c.to_cap, x2 = x * x;
  float near = product * c.to2 * fmaf(x2, fmaf(x2, fmaf(x2, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), 1.f);
  asm volatile("" : "+v"(near));            // chosen, not branched to: branches around 16 of them would cost dk and dv their registers
  return fabsf(x) < 0.25f ? near : far;
}
__device__ __forceinline__ float biased(float s, float slope2, float rel, int r) { return fmaf(-slope2, fabsf(rel - (float)row_of(r)), s); }

// A lane's row of the 32 of its wavefront: row first + lane % 32; those behind the last see what it sees (they are not stored)
template <class T, int D>
struct QueryRow {
  s8 q[D / 16];
  int row, token, head, pos;
  uint32_t word, raw;                       // as the comparisons want it, and as it is
  float slope2;
  __device__ __forceinline__ void start(const AttnCall &c, int b, int h, int first, int lane) {
    row = first + (lane & 31);
    const int r = row < c.rows ? row : c.rows - 1;
    token = divide(c.by_group, r);
    head = h * c.group + r - token * c.group;
    pos = token + c.offset;
    raw = c.q_words ? c.q_words[(int64_t)b * c.q_tile_count * ATTN_TILE + token] & ~1u : 0;
    word = query_word(raw);
    slope2 = c.slopes ? c.slopes[head] * 1.44269504088896341f : 0.f;
  }
  // operands straight from memory, 16 bytes a row and load: for few rows
  __device__ __forceinline__ void operands(const AttnCall &c, int b, int lane) {
    const uint16_t *p = c.q.p + b * c.q.batch + token * c.q.token + head * c.q.head;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const int d = k * 16 + (lane >> 5) * 8;
      q[k] = d < c.dim ? *(const s8 *)(p + d) : s8{};
    }
  }
};
// A wavefront's 32 rows of queries or dy to its own memory: whole rows a load
template <int D>
__device__ __forceinline__ void bring_rows(const AttnCall &c, const AttnInput &in, const Place &p, int first, uint32_t lds, int lane) {
  RowFeed<D, 32, 1> feed;
  feed.start(in, p.b, p.h * c.group);
  feed.once(c, first, lds, lane);
}

// A running softmax over blocks of 32 keys: reference (powers of two) and sum.  The reference follows the maximum only when that has grown by more than
// 2^8: until then weights are up to 256, which 16-bit floats hold as exactly as smaller ones, and nothing has to be rescaled.
//
// Until the exponential a score stays what it costs least to get: the product; with a cap 1 / (1 + exp(2 x)) (capped()), which falls as the score grows;
// with a bias the score itself.  weight = exp2(value * unit() + base() - reference).
template <class T, int D, int CAP, int SLOPE>
struct Softmax {
  enum { LEAST = CAP && !SLOPE };           // values fall as scores grow
  f16 o[D / 32];
  float top, sum;
  __device__ __forceinline__ void start() {
    top = LOWEST;
    sum = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f16{};
  }
  static __device__ __forceinline__ float unit(const AttnCall &c) { return SLOPE ? 1.f : CAP ? -2.f * c.cap2 : c.to2; }
  static __device__ __forceinline__ float base(const AttnCall &c) { return LEAST ? c.cap2 : 0.f; }
  static __device__ __forceinline__ float more(float a, float b) { return LEAST ? fminf(a, b) : fmaxf(a, b); }

  static __device__ __forceinline__ f16 products(const QueryRow<T, D> &row, const lds_char *keys, int first, int lane) {
    f16 s = {};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) s = T::mfma(row_fragment<D>(keys, first, k, lane), row.q[k], s);
    return s;
  }
  // values from the products with the keys k0 + row_of(r)
  static __device__ __forceinline__ void values_of(const AttnCall &c, const QueryRow<T, D> &row, int k0, f16 &s) {
    if (!CAP && !SLOPE) return;
    const float rel = SLOPE ? (float)(row.pos - k0) : 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (LEAST) {
        s[r] = __builtin_amdgcn_rcpf(1.f + exp2_(s[r] * c.tanh2));
      } else {
        float share;
        s[r] = biased(capped<CAP>(c, s[r], share), row.slope2, rel, r);
      }
    }
  }
  // those of hidden keys become the value of no weight
  static __device__ __forceinline__ void hide(const AttnCall &c, const QueryRow<T, D> &row, const Visit &now, uint32_t there, int k0, int lane, f16 &s) {
    const uint32_t seen = seen_keys(c, now, there, k0, row.pos, row.word, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = where_seen(seen, r, s[r], LEAST ? 0x7f800000u : 0xff800000u);
  }
  static __device__ __forceinline__ float most_of(const f16 &s) {
    float m = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) m = more(m, s[r]);
    return m;
  }
  // brings the reference to where the weights of values up to `most` are at most 2^8
  __device__ __forceinline__ void follow(const AttnCall &c, float most) {
    const float to = both_max(fmaf(most, unit(c), base(c)));
    if (__any(to > top + 8.f)) {
      const float up = fmaxf(top, to), f = exp2_(top - up);
      top = up;
      sum *= f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] *= f;
    }
  }
  // the weights of 32 keys, and the sums of their values (the rows from `first` on)
  __device__ __forceinline__ void add(const AttnCall &c, f16 &s, const lds_char *values, int first, int lane) {
    const float less = base(c) - top;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = exp2_(SLOPE ? s[r] + less : fmaf(s[r], unit(c), less));
      sum += s[r];
    }
    const s8 p[2] = {pack8<T>(s, 0), pack8<T>(s, 8)};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] = T::mfma(column_fragment<D>(values, first + k * 16, d, lane), p[k], o[d]);
  }
};

// A wavefront's results, 32 rows (in lanes) of N blocks of 32 columns (the first: d0), turned round in shared memory, two blocks at a time, so that they
// leave as rows: 8 elements a lane
constexpr int turn_bytes(int blocks) { return 32 * (blocks >= 2 ? 68 : 36) * 4; }
template <int N, class F>
__device__ __forceinline__ void by_rows(lds_char *own, const f16 (&v)[N], int d0, int lane, F f) {
  constexpr int B = N >= 2 ? 2 : 1, PITCH = B * 32 + 4, EACH = B * 4;       // EACH: lanes a row
  const int h4 = (lane >> 5) * 4;
#pragma unroll
  for (int at = 0; at < N; at += B) {
#pragma unroll
    for (int d = 0; d < B; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(__attribute__((address_space(3))) f4 *)(own + ((lane & 31) * PITCH + d * 32 + g * 8 + h4) * 4) =
            f4{v[at + d][g * 4], v[at + d][g * 4 + 1], v[at + d][g * 4 + 2], v[at + d][g * 4 + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < EACH / 2; ++i) {
      const int row = i * (64 / EACH) + lane / EACH, d = lane % EACH * 8;
      const __attribute__((address_space(3))) f4 *p = (const __attribute__((address_space(3))) f4 *)(own + (row * PITCH + d) * 4);
      f(row, d0 + at * 32 + d, p[0], p[1]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// Two wavefronts have parts of the same sums of N * 2 blocks.  Each keeps half of them (the second wavefront the second half) and gives the other half
// to the other by shared memory: `give` before a barrier, `take` behind it
template <int N>
__device__ __forceinline__ void give(lds_char *at, const f16 (&v)[2 * N], f16 (&mine)[N], bool second, int lane) {
#pragma unroll
  for (int d = 0; d < N; ++d) {
    const f16 other = second ? v[d] : v[N + d];
    mine[d] = second ? v[N + d] : v[d];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(__attribute__((address_space(3))) f4 *)(at + ((d * 4 + g) * 64 + lane) * 16) = f4{other[g * 4], other[g * 4 + 1], other[g * 4 + 2], other[g * 4 + 3]};
  }
}
template <int N>
__device__ __forceinline__ void take(const lds_char *at, f16 (&mine)[N], float f, float f_other, int lane) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f4 v = *(const __attribute__((address_space(3))) f4 *)(at + ((d * 4 + g) * 64 + lane) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[d][g * 4 + e] = fmaf(mine[d][g * 4 + e], f, v[e] * f_other);
    }
}
// 8 elements of a row of the results
template <class T>
__device__ __forceinline__ void store8(uint16_t *p, int d, int width, f4 a, f4 b) {
  const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  if (d + 8 <= width) {
    typedef uint32_t u4_anywhere __attribute__((ext_vector_type(4), aligned(2)));
    u4_anywhere w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)T::down(v[2 * i]) | ((uint32_t)T::down(v[2 * i + 1]) << 16);
    *(u4_anywhere *)(p + d) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (d + i < width) p[d + i] = T::down(v[i]);
  }
}
// what rounding took from them
template <class T>
__device__ __forceinline__ void store8_low(uint16_t *p, int d, int width, f4 a, f4 b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] -= T::up(T::down(a[i]));
    b[i] -= T::up(T::down(b[i]));
  }
  store8<T>(p, d, width, a, b);
}

// ---------------------------------------------------------------------------------------------- forward
// 32 rows a wavefront; two wavefronts a SIMD (three with rows of 64), of different workgroups, so that one's products run beside another's
// exponentials.  PARTS = 1: a workgroup has 128 rows.  2: it has 64, each wavefront half of the keys of a tile; the sums meet at the end.  Every tile is read
// for half as many rows then, but a workgroup takes half as long, and the longest one is what a small call waits for (2 x 515 tokens, 6 heads of 72, everything:
// 23 us with 128 rows, 17 with 64).
template <class T, int D, int CAP, int SLOPE, int PARTS>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) k_forward(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WAVES = 4, BLOCKS = WAVES / PARTS, N = D / 32 / PARTS;      // blocks of rows; blocks of columns that a wavefront stores
  typedef TileFeed<D, WAVES> Feed;
  typedef Softmax<T, D, CAP, SLOPE> Soft;
  constexpr int TURN = WAVES * turn_bytes(N), MEET = PARTS == 2 ? WAVES * N * 4096 : 0;
  __shared__ __attribute__((aligned(1024))) char shared[Feed::BYTES > TURN + MEET ? Feed::BYTES : TURN + MEET];
  __shared__ float tops[WAVES][32], sums[WAVES][32];
  lds_char *lds = (lds_char *)shared;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave / BLOCKS;
  const Place p = place_of(c, blockIdx.x, true);
  const int row0 = p.tile * (BLOCKS * 32), wave_row = row0 + wave % BLOCKS * 32, h4 = (lane >> 5) * 4;
  // the queries come by the second slot, a wavefront's to its own part
  const int mine = Feed::SLOT + wave * Shape<D>::bytes(32);
  static_assert(WAVES * Shape<D>::bytes(32) <= Feed::SLOT, "a slot holds the rows");
  bring_rows<D>(c, c.q, p, wave_row, lds0 + mine, lane);
  Feed feed;
  feed.start(c, p, wave, lane);
  QueryRow<T, D> row;
  row.start(c, p.b, p.h, wave_row, lane);
  KeyWalk<BLOCKS * 32> walk;
  walk.start(c, p.b, row0, wave_row, row.raw, p.split, c.splits, c.tiles, lane);
  Visit next = walk.next(c, lane);
  if (next.tile >= 0) feed.load(next.tile, lds0, wave, lane);
  Soft soft;
  soft.start();
  waited<0>();
#pragma unroll
  for (int k = 0; k < D / 16; ++k) row.q[k] = row_fragment<D>(lds + mine, 0, k, lane);

  int slot = 0;
  while (next.tile >= 0) {
    const Visit now = next;
    next = walk.next(c, lane);
    arrived();                              // this tile is there, and the other slot has been read by everybody
    lds_char *here = lds + slot * Feed::SLOT, *values = here + Feed::VALUES;
    if (now.some_none) {
      Feed::clear(here, values, tid);
      arrived();
    }
    slot ^= 1;
    if (next.tile >= 0) feed.load(next.tile, lds0 + slot * Feed::SLOT, wave, lane);
    if (!now.run) continue;
    const int first = PARTS == 2 ? part * 32 : 0, k0 = now.tile * ATTN_TILE + first + h4;
    lds_word *words = (lds_word *)(here + Feed::WORDS) + first + (lane & 31);
    f16 s = Soft::products(row, here, first, lane);
    if (PARTS == 2) {
      Soft::values_of(c, row, k0, s);
      if (now.masked()) Soft::hide(c, row, now, words[0], k0 - h4, lane, s);
      soft.follow(c, Soft::most_of(s));
      soft.add(c, s, values, first, lane);
    } else {
      f16 t = Soft::products(row, here, 32, lane);
      Soft::values_of(c, row, k0, s);
      Soft::values_of(c, row, k0 + 32, t);
      if (now.masked()) {
        Soft::hide(c, row, now, words[0], k0 - h4, lane, s);
        Soft::hide(c, row, now, words[32], k0 - h4 + 32, lane, t);
      }
      soft.follow(c, Soft::more(Soft::most_of(s), Soft::most_of(t)));
      soft.add(c, s, values, 0, lane);
      soft.add(c, t, values, 32, lane);
    }
  }

  arrived();
  float sum = both_sum(soft.sum), top = soft.top;
  f16 o[N];
  if constexpr (PARTS == 2) {
    const int other = wave ^ BLOCKS;
    if (lane < 32) {
      tops[wave][lane] = top;
      sums[wave][lane] = sum;
    }
    give<N>(lds + TURN + wave * (N * 4096), soft.o, o, part == 1, lane);
    __syncthreads();
    const float far = tops[other][lane & 31];
    top = fmaxf(top, far);
    const float f = exp2_(soft.top - top), g = exp2_(far - top);
    sum = fmaf(sum, f, sums[other][lane & 31] * g);
    take<N>(lds + TURN + other * (N * 4096), o, f, g, lane);
  } else {
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = soft.o[d];
  }
  lds_char *own = lds + wave * turn_bytes(N);
  const int d0 = part * (N * 32);
  if (c.splits > 1) {
    const int64_t at = ((int64_t)p.split * c.batch * c.kv_heads + p.hb) * c.rows + wave_row;
    if (part == 0 && lane < 32 && row.row < c.rows) {
      c.part2[(at + lane) * 2] = top;
      c.part2[(at + lane) * 2 + 1] = sum;
    }
    by_rows(own, o, d0, lane, [&](int i, int d, f4 a, f4 b) {
      if (wave_row + i >= c.rows) return;
      float *out = c.part + (at + i) * c.width4 + d;
      if (d < c.width4) *(f4 *)out = a;
      if (d + 4 < c.width4) *(f4 *)(out + 4) = b;
    });
    return;
  }
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  if (c.lse && part == 0 && lane < 32 && row.row < c.rows) c.lse[(int64_t)p.hb * c.rows_pad + row.row] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
#pragma unroll
  for (int d = 0; d < N; ++d) o[d] *= f;
  by_rows(own, o, d0, lane, [&](int i, int d, f4 a, f4 b) {
    const int r = wave_row + i, token = divide(c.by_group, r), head = p.h * c.group + r - token * c.group;
    if (r >= c.rows) return;
    store8<T>(c.y.p + p.b * c.y.batch + token * c.y.token + head * c.y.head, d, c.width, a, b);
    if (c.low) store8_low<T>(c.low + (((int64_t)p.b * c.tokens + token) * (c.kv_heads * c.group) + head) * c.width, d, c.width, a, b);
  });
#endif
}

// Up to 32 rows (the heads of a group for a token or a few) over many keys: bound by reading the keys and values.  Each wavefront has all rows, its
// own keys and its own shared memory, 32 keys at a time, and waits for nobody; the wavefronts' parts are joined at the end.  8 answers of 32,768 keys, 32
// heads of 128, 8 of keys: 191 us, 5.6 TB/s (what a read alone reaches); 64 answers of 1,024 keys on average, 16 heads of 64: 59 us, 4.4 TB/s.
template <class T, int D, int CAP, int SLOPE>
__global__ void __launch_bounds__(256) k_forward_few(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WAVES = 4;
  typedef KeyFeed<D, 32, 1> Feed;
  constexpr int OWN = 4 * Feed::BYTES;      // two steps of keys and values; behind the loop 32 rows of D sums
  __shared__ __attribute__((aligned(1024))) char shared[WAVES * OWN];
  __shared__ float tops[WAVES][32], sums[WAVES][32];
  lds_char *lds = (lds_char *)shared;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  lds_char *own = lds + wave * OWN;
  const uint32_t own0 = (uint32_t)(uintptr_t)own;
  const Place p = place_of(c, blockIdx.x, false);
  QueryRow<T, D> row;
  row.start(c, p.b, p.h, 0, lane);
  row.operands(c, p.b, lane);
  Feed kf, vf;
  kf.start(c.k, p.b, p.h, c.keys, c.dim, 0, lane);
  vf.start(c.v, p.b, p.h, c.keys, c.dim, 0, lane);
  const uint32_t *words = c.k_words ? c.k_words + (int64_t)p.b * c.tiles * ATTN_TILE : nullptr;
  KeyWalk<32> walk;
  walk.start(c, p.b, 0, 0, row.raw, p.split * WAVES + wave, c.splits * WAVES, c.tiles, lane);
  typedef Softmax<T, D, CAP, SLOPE> Soft;
  Soft soft;
  soft.start();

  int slot = 0, half = 0;
  Visit next = walk.next(c, lane);
  if (next.tile >= 0) {
    kf.load(next.tile * ATTN_TILE, own0, 0);
    vf.load(next.tile * ATTN_TILE, own0 + Feed::BYTES, 0);
  }
  while (next.tile >= 0) {
    const Visit now = next;
    const int k0 = now.tile * ATTN_TILE + half * 32;
    half ^= 1;
    if (half == 0 || k0 + 32 >= c.keys) {
      half = 0;
      next = walk.next(c, lane);
    }
    lds_char *here = own + slot * 2 * Feed::BYTES;
    slot ^= 1;
    if (next.tile >= 0) {
      const int k = next.tile * ATTN_TILE + half * 32;
      kf.load(k, own0 + slot * 2 * Feed::BYTES, 0);
      vf.load(k, own0 + slot * 2 * Feed::BYTES + Feed::BYTES, 0);
      waited<2 * Feed::LOADS>();
    } else {
      waited<0>();
    }
    if (now.some_none) {
      clear_none<D, 32, 64>(here + Feed::BYTES, words + k0, lane);
      waited<0>();
    }
    f16 s = Soft::products(row, here, 0, lane);
    Soft::values_of(c, row, k0 + (lane >> 5) * 4, s);
    if (now.masked()) Soft::hide(c, row, now, words ? words[k0 + (lane & 31)] : 0, k0, lane, s);
    soft.follow(c, Soft::most_of(s));
    soft.add(c, s, here + Feed::BYTES, 0, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the slot has been read: the next loads go there
  }

  constexpr int PITCH = D + 4;              // floats: 32 rows of it in a wavefront's own memory
  static_assert(32 * PITCH * 4 <= OWN, "the sums of a wavefront");
  const float total = both_sum(soft.sum);
  const int h4 = (lane >> 5) * 4;
  if (lane < 32) {
    tops[wave][lane] = soft.top;
    sums[wave][lane] = total;
  }
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(__attribute__((address_space(3))) f4 *)(own + ((lane & 31) * PITCH + d * 32 + g * 8 + h4) * 4) =
          f4{soft.o[d][g * 4], soft.o[d][g * 4 + 1], soft.o[d][g * 4 + 2], soft.o[d][g * 4 + 3]};
  __syncthreads();
  const int live = c.rows < 32 ? c.rows : 32;
  for (int i = tid; i < live * (D / 8); i += 256) {
    const int r = i / (D / 8), d = i % (D / 8) * 8;
    float top = tops[0][r];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w][r]);
    float sum = 0.f;
    f4 v = f4{0.f, 0.f, 0.f, 0.f}, u = v;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float f = exp2_(tops[w][r] - top);
      const __attribute__((address_space(3))) f4 *part = (const __attribute__((address_space(3))) f4 *)(lds + w * OWN + (r * PITCH + d) * 4);
      sum += sums[w][r] * f;
      v += part[0] * f;
      u += part[1] * f;
    }
    if (c.splits > 1) {
      const int64_t at = ((int64_t)p.split * c.batch * c.kv_heads + p.hb) * c.rows + r;
      if (d == 0) {
        c.part2[at * 2] = top;
        c.part2[at * 2 + 1] = sum;
      }
      if (d < c.width4) *(f4 *)(c.part + at * c.width4 + d) = v;
      if (d + 4 < c.width4) *(f4 *)(c.part + at * c.width4 + d + 4) = u;
      continue;
    }
    const int token = divide(c.by_group, r), head = p.h * c.group + r - token * c.group;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    if (c.lse && d == 0) c.lse[(int64_t)p.hb * c.rows_pad + r] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
    store8<T>(c.y.p + p.b * c.y.batch + token * c.y.token + head * c.y.head, d, c.width, v * f, u * f);
    if (c.low) store8_low<T>(c.low + (((int64_t)p.b * c.tokens + token) * (c.kv_heads * c.group) + head) * c.width, d, c.width, v * f, u * f);
  }
#endif
}

// ---------------------------------------------------------------------------------------------- backward
// p and ds of a score from the products q.k and dy.v.  less: lse (with a bias, and it) in powers of two, less cap2 with a cap (CAP = 1); delta: dy.y, four times it with a
// cap, where ds = p share (1 - share) (4 dy.v - 4 delta)
template <int CAP>
__device__ __forceinline__ void gradient(const AttnCall &c, float product, float dp, float less, float delta, float &p, float &ds) {
  if (CAP == 2) {
    float share;
    p = exp2_(capped<CAP>(c, product, share) - less);
    ds = p * fmaf(-share, share, share) * fmaf(dp, 4.f, -delta);
  } else if (CAP) {
    const float share = __builtin_amdgcn_rcpf(1.f + exp2_(product * c.tanh2));
    p = exp2_(fmaf(share, -2.f * c.cap2, -less));
    ds = p * fmaf(-share, share, share) * fmaf(dp, 4.f, -delta);
  } else {
    p = exp2_(fmaf(product, c.to2, -less));
    ds = p * (dp - delta);
  }
}

// A block of 32 keys whose lifted ds pass 2^15: from here on the lane's row has less of the lift, in its weights, this block and the sums, so that the largest lies between 2^13 and
// 2^14.  How much less is kept for dk (rows of 32 together, AttnRows::lowered).  A bound that is known beforehand, |dy| times the largest |v|, would cost a launch of its own and half of the lift in
// calls that need none taken away.  Time, 8,192 tokens, 32 heads of 128, 8 of keys: dq 870 us for 805 without, capped 973 for 925, dk and dv 1,207 for 1,195, capped
// 1,272 for 1,262; 4 x 1,024 tokens of 64: 36 for 33.5 and 43.6 for 43.
template <int D>
__device__ __forceinline__ void lower(f16 &ds, f16 (&sums)[D / 32], float &less, int &lowered) {
  const auto largest = [](float a, float b, float c) {        // written out: the compiler makes values that passed a mask canonical first, one more operation each
    float m;
    asm("v_max3_f32 %0, |%1|, |%2|, |%3|" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
  };
  float m = ds[0];
#pragma unroll
  for (int r = 1; r < 15; r += 2) m = largest(m, ds[r], ds[r + 1]);
  m = both_max(largest(m, ds[15], ds[15]));
  if (__any(m >= 32768.f)) {
    const int e = m >= 32768.f ? __builtin_amdgcn_frexp_expf(m) : 0, n = e > 14 ? e - 14 : 0;       // infinities: 0, they stay
    less += (float)n;
    lowered += n;
#pragma unroll
    for (int r = 0; r < 16; ++r) ds[r] = ldexpf(ds[r], -n);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums[d][r] = ldexpf(sums[d][r], -n);
  }
}
// sums without their lift
template <int N>
__device__ __forceinline__ void take_down(f16 (&sums)[N], int by) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) sums[d][r] = ldexpf(sums[d][r], by);
}

// delta = dy.y of a wavefront's 32 rows, whose dy lie at `dys`, to `out`.  y is taken with what its rounding took from it: where few keys share a row, dy.v and
// delta are near each other, and 2^-9 of y would be 1.5 times the error that the gradients have otherwise (17 tokens in bfloat16, dk: 3.7e-3
// without, 2.4e-3 with).  A row by as many lanes as it has chunks.
template <class T, int D, int ROWS>
struct Deltas {
  typedef Shape<D> S;
  typedef s8 s8_anywhere __attribute__((aligned(2)));
  enum { EACH = S::CHUNKS, AT_ONCE = 64 / EACH, N = ROWS / AT_ONCE };
  s8 y[N], low[N];
  // asks for ROWS rows from `first` on
  __device__ __forceinline__ void start(const AttnCall &c, const Place &p, int first, int lane) {
    const int d = lane % EACH * 8;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = first + i * AT_ONCE + lane / EACH, r = row < c.rows ? row : c.rows - 1, token = divide(c.by_group, r), head = p.h * c.group + r - token * c.group;
      const uint16_t *a = c.y_in.p + p.b * c.y_in.batch + token * c.y_in.token + head * c.y_in.head;
      const uint16_t *b = c.low + (((int64_t)p.b * c.tokens + token) * (c.kv_heads * c.group) + head) * c.width;
      if (c.width % 8 == 0) {               // chunks behind the last: left out of the sum
        const int at = d < c.width ? d : 0;
        y[i] = *(const s8_anywhere *)(a + at);
        low[i] = *(const s8_anywhere *)(b + at);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool in = d + e < c.width;
          y[i][e] = in ? (short)a[d + e] : (short)0;
          low[i][e] = in ? (short)b[d + e] : (short)0;
        }
      }
    }
  }
  // their dy are the rows from `first` on of `dys`
  __device__ __forceinline__ void finish(const AttnCall &c, const lds_char *dys, int first, float *out, int lane) const {
    const int chunk = lane % EACH;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = first + i * AT_ONCE + lane / EACH;
      const s8 dy = *(const __attribute__((address_space(3))) s8 *)(dys + S::row_at(row) + ((uint32_t)chunk ^ S::swizzle(row)) * 16);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(T::up((uint16_t)dy[e]), T::up((uint16_t)y[i][e]) + T::up((uint16_t)low[i][e]), sum);
      if (chunk * 8 >= c.width) sum = 0.f;
#pragma unroll
      for (int x = EACH / 2; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
      if (chunk == 0) out[i * AT_ONCE + lane / EACH] = sum;
    }
  }
};

// How the sums of a sequence's tiles of keys are shared out for dk and dv: each tile by how many blocks of rows see it, in parts as equal as their number
// allows, the longest first.  Half of the slots are used where that leaves short parts: what is saved is their sums' way through memory (4,096 packed
// tokens, 32 heads of 128, 8 of keys: 512 parts 124 + 12 us, 1,024 parts 122 + 25), while longer ones fill the GPU better in twice as many (4,096 tokens in one
// document 400 + 14, 347 + 24).  A workgroup of its own, which is done long before the others.
enum { SHARE_COSTS = ATTN_SHARE_QUERIES * 16, SHARE_BYTES = SHARE_COSTS + ATTN_SHARE_TILES * 4 + 16 };
__device__ __forceinline__ void share_keys(const AttnCall &c, int b, lds_char *lds) {
  __attribute__((address_space(3))) i4 *queries = (__attribute__((address_space(3))) i4 *)lds;
  __attribute__((address_space(3))) int *cost = (__attribute__((address_space(3))) int *)(lds + SHARE_COSTS), *total = cost + ATTN_SHARE_TILES;
  const int n = c.share_tiles, each = c.share_keys / ATTN_TILE;
  if (c.k_words)
    for (int i = threadIdx.x; i < c.q_tile_count; i += 256) queries[i] = *(const i4 *)&c.q_tiles[(int64_t)b * c.q_tile_count + i];
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int k0 = i * c.share_keys, k1 = k0 + c.share_keys - 1 < c.keys ? k0 + c.share_keys - 1 : c.keys - 1;
    Range k{INT32_MAX, -1, 0};
    if (c.k_words)
      for (int j = i * each; j < (i + 1) * each && j < c.tiles; ++j) {
        const AttnTile x = c.k_tiles[(int64_t)b * c.tiles + j];
        k = join(k, x);
        k.flags |= x.flags & ATTN_SOME_PREFIX;
      }
    int seen = 0;
    for (int j = 0; j < c.q_tile_count; ++j) {
      const i4 x = c.k_words ? queries[j] : i4{};
      seen += sees(c, j * ATTN_TILE + c.offset, j * ATTN_TILE + ATTN_TILE - 1 + c.offset, Range{x[0], x[1], x[2]}, k0, k1, k).some;
    }
    cost[i] = seen < 1 ? 1 : seen * c.share_unit;
  }
  __syncthreads();
  int64_t all = 0;
  for (int j = 0; j < n; ++j) all += cost[j];
  const int half = c.share_slots / 2 > n ? c.share_slots / 2 : n, limit = all <= half * c.share_short ? half : c.share_slots;
  // the least length of a part with which there are enough of them
  int low = c.share_least, high = c.q_tile_count * c.share_unit > c.share_least ? c.q_tile_count * c.share_unit : c.share_least;
  while (low < high) {
    const int length = (low + high) / 2;
    __syncthreads();
    if (threadIdx.x == 0) *total = 0;
    __syncthreads();
    int parts = 0;
    for (int i = threadIdx.x; i < n; i += 256) parts += (cost[i] + length - 1) / length;
    __hip_atomic_fetch_add(total, parts, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __syncthreads();
    if (*total <= limit) high = length;
    else low = length + 1;
  }
  __syncthreads();
  const auto parts_of = [&](int cost) { return (cost + low - 1) / low; };
  const auto length_of = [&](int cost) { return (cost + parts_of(cost) - 1) / parts_of(cost); };
  AttnShare *shares = c.shares + (int64_t)b * c.share_slots;
  int used = 0;
  for (int j = 0; j < n; ++j) used += parts_of(cost[j]);
  for (int i = threadIdx.x; i < n; i += 256) {
    const int mine = cost[i], parts = parts_of(mine), length = length_of(mine);
    int before = 0, slot = 0;
    for (int j = 0; j < n; ++j) {
      const int far = length_of(cost[j]), p = parts_of(cost[j]);
      before += far > length || (far == length && j < i) ? p : 0;
      slot += j < i ? p : 0;
    }
    for (int k = 0; k < parts; ++k) shares[before + k] = AttnShare{i, k, parts, slot + k};
    c.tile_slots[(int64_t)b * n + i] = AttnSlots{slot, parts};
  }
  for (int i = used + threadIdx.x; i < c.share_slots; i += 256) shares[i] = AttnShare{-1, 0, 1, 0};
}

// PARTS as in k_forward.  FINE: ds enters its product with what its rounding took, a second product; so in dk and dv, and p as well.  Otherwise gradients are off by 1.4 times
// what their own rounding makes, with it by hardly more than that.  Taken where a call leaves most compute units idle and sums are too few for
// errors to be alike: 17 tokens, 4 heads of 64, dq + dk and dv 8.5 + 7.6 us without, 8.8 + 8.2 with; 2 x 515 tokens, 6 heads of 72 19.0 + 21.2, 19.1 + 23.1; 512 tokens, 32
// heads of 128, 8 of keys (256 workgroups: not taken) 20.0 + 22.8, 21.8 + 29.0.
template <class T, int D, int CAP, int SLOPE, int PARTS, int FINE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 ? 3 : 2))) k_dq(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WAVES = 4, BLOCKS = WAVES / PARTS, N = D / 32 / PARTS;
  typedef TileFeed<D, WAVES> Feed;
  constexpr int TURN = WAVES * turn_bytes(N), MEET = PARTS == 2 ? WAVES * N * 4096 : 0;
  static_assert((int)SHARE_BYTES <= (int)Feed::BYTES, "shared memory holds what the shares are worked out from");
  __shared__ float deltas[BLOCKS][32];
  __shared__ int most[WAVES];
  __shared__ __attribute__((aligned(1024))) char shared[Feed::BYTES > TURN + MEET ? Feed::BYTES : TURN + MEET];
  lds_char *lds = (lds_char *)shared;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave / BLOCKS, block = wave % BLOCKS;
  if ((int)blockIdx.x < c.share_groups) return share_keys(c, blockIdx.x, lds);
  const Place p = place_of(c, blockIdx.x - c.share_groups, true);
  const int row0 = p.tile * (BLOCKS * 32), wave_row = row0 + block * 32, h4 = (lane >> 5) * 4;
  // dy comes by the second slot, a wavefront's rows to its own part
  const int mine = Feed::SLOT + wave * Shape<D>::bytes(32);
  static_assert(WAVES * Shape<D>::bytes(32) <= Feed::SLOT, "a slot holds the rows");
  bring_rows<D>(c, c.dy, p, wave_row, lds0 + mine, lane);
  Feed feed;
  feed.start(c, p, wave, lane);
  QueryRow<T, D> row;
  row.start(c, p.b, p.h, wave_row, lane);
  row.operands(c, p.b, lane);
  constexpr int SHARE = 32 / PARTS;         // rows whose delta a wavefront works out
  Deltas<T, D, SHARE> known;
  known.start(c, p, wave_row + part * SHARE, lane);
  const bool there = row.row < c.rows;
  const float lse = c.lse[(int64_t)p.hb * c.rows_pad + (there ? row.row : c.rows - 1)];
  KeyWalk<BLOCKS * 32> walk;
  walk.start(c, p.b, row0, wave_row, row.raw, 0, 1, c.tiles, lane);
  Visit next = walk.next(c, lane);
  if (next.tile >= 0) feed.load(next.tile, lds0, wave, lane);
  waited<0>();
  s8 dy[D / 16];
#pragma unroll
  for (int k = 0; k < D / 16; ++k) dy[k] = row_fragment<D>(lds + mine, 0, k, lane);
  known.finish(c, lds + mine, part * SHARE, &deltas[block][part * SHARE], lane);
  if (PARTS == 2) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  float less = (CAP == 1 ? lse - c.cap2 : lse) - T::LIFT;
  const float delta = CAP ? 4.f * deltas[block][lane & 31] : deltas[block][lane & 31];
  if (part == 0 && lane < 32 && row.row < c.rows_pad) {
    AttnRows &block = c.row_data[(int64_t)p.hb * (c.rows_pad / 32) + (row.row >> 5)];
    block.less[lane] = there ? less : INFINITY;
    block.delta[lane] = delta;
    block.word[lane] = there ? row.word : ATTN_NOBODY;
    block.slope2[lane] = row.slope2;
    block.pos[lane] = row.pos;
    if (c.k_words && lane == 0) block.documents = AttnTile{walk.wave_docs.first, walk.wave_docs.last, walk.wave_docs.flags, 0};
  }
  f16 dq[D / 32];
  int lowered = 0;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dq[d] = f16{};

  int slot = 0;
  while (next.tile >= 0) {
    const Visit now = next;
    next = walk.next(c, lane);
    arrived();
    lds_char *keys = lds + slot * Feed::SLOT, *values = keys + Feed::VALUES;
    lds_word *words = (lds_word *)(keys + Feed::WORDS) + (lane & 31);
    if (now.some_none) {
      Feed::clear(keys, keys, tid);
      arrived();
    }
    slot ^= 1;
    if (next.tile >= 0) feed.load(next.tile, lds0 + slot * Feed::SLOT, wave, lane);
    if (!now.run) continue;
#pragma unroll
    for (int half = 0; half < 2 / PARTS; ++half) {
      // 8,192 tokens, 32 heads of 128, 8 of keys, capped: 990 us, without it 1,035; without a cap 875 and 835, but in float16, where lower() parts the halves, 860 and 944
      if (CAP || T::LIFT != 0) __builtin_amdgcn_sched_barrier(0);
      const int b = PARTS == 2 ? part : half, k0 = now.tile * ATTN_TILE + b * 32 + h4;
      f16 s = {}, dp = {};
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        s = T::mfma(row_fragment<D>(keys, b * 32, k, lane), row.q[k], s);
        dp = T::mfma(row_fragment<D>(values, b * 32, k, lane), dy[k], dp);
      }
      const float rel = SLOPE ? (float)(row.pos - k0) : 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float weight, ds;
        gradient<CAP>(c, s[r], dp[r], SLOPE ? fmaf(row.slope2, fabsf(rel - (float)row_of(r)), less) : less, delta, weight, ds);
        dp[r] = ds;
      }
      if (now.masked()) {
        const uint32_t seen = seen_keys(c, now, words[b * 32], k0 - h4, row.pos, row.word, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = where_seen(seen, r, dp[r], 0);
      }
      if constexpr (T::LIFT != 0) lower<D>(dp, dq, less, lowered);
      const s8 ds[2] = {pack8<T>(dp, 0), pack8<T>(dp, 8)};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const s8 low = FINE ? pack8_low<T>(dp, ds[k], k * 8) : s8{};
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const s8 key = column_fragment<D>(keys, b * 32 + k * 16, d, lane);
          dq[d] = T::mfma(key, ds[k], dq[d]);
          if (FINE) dq[d] = T::mfma(key, low, dq[d]);
        }
      }
    }
  }
  arrived();
  if constexpr (T::LIFT != 0) {
    take_down<D / 32>(dq, lowered - T::LIFT);
#pragma unroll
    for (int x = 16; x >= 1; x >>= 1) {
      const int other = __shfl_xor(lowered, x);
      lowered = other > lowered ? other : lowered;
    }
    if (lane == 0) most[wave] = lowered;
  }
  f16 sum[N];
  if constexpr (PARTS == 2) {
    give<N>(lds + TURN + wave * (N * 4096), dq, sum, part == 1, lane);
    __syncthreads();
    if (T::LIFT != 0 && most[wave ^ BLOCKS] > lowered) lowered = most[wave ^ BLOCKS];
    take<N>(lds + TURN + (wave ^ BLOCKS) * (N * 4096), sum, c.scale, c.scale, lane);
  } else {
#pragma unroll
    for (int d = 0; d < N; ++d) sum[d] = dq[d] * c.scale;
  }
  if (T::LIFT != 0 && part == 0 && lane == 0 && wave_row < c.rows_pad) c.row_data[(int64_t)p.hb * (c.rows_pad / 32) + (wave_row >> 5)].lowered = lowered;
  by_rows(lds + wave * turn_bytes(N), sum, part * (N * 32), lane, [&](int i, int d, f4 a, f4 b) {
    const int r = wave_row + i, token = divide(c.by_group, r), head = p.h * c.group + r - token * c.group;
    if (r < c.rows) store8<T>(c.dq.p + p.b * c.dq.batch + token * c.dq.token + head * c.dq.head, d, c.width, a, b);
  });
#endif
}

// Blocks of ROWS rows (32 of a wavefront's own: those from `own` on) that see some of a workgroup's KEYS keys, as KeyWalk
template <int KEYS, int ROWS>
struct RowWalk {
  int group_from, group_to, wave_from, wave_to;           // keys
  Range group_docs, wave_docs;
  const AttnRows *rows;                     // what the rows' documents are, or null
  int own, first, step, at, end;
  uint64_t visit, mine, documents, order, none;
  // word: of the lane's key
  __device__ __forceinline__ void start(const AttnCall &c, const Place &p, int group_key, int wave_key, uint32_t word, int own_, int first_, int step_, int end_, int lane) {
    own = own_;
    group_from = group_key;
    group_to = group_key + KEYS - 1 < c.keys ? group_key + KEYS - 1 : c.keys - 1;
    wave_from = wave_key < c.keys ? wave_key : c.keys - 1;
    wave_to = wave_key + 31 < c.keys ? wave_key + 31 : c.keys - 1;
    first = first_;
    step = step_;
    at = 0;
    end = end_;
    rows = c.k_words ? c.row_data + (int64_t)p.hb * (c.rows_pad / 32) : nullptr;
    const Known x = documents_of(lane);
    if (rows) {
      group_docs = keys_of<KEYS / 64>(c.k_tiles + (int64_t)p.b * c.tiles, group_from, group_to);
      wave_docs = range_of(word);
    }
    choose(c, x, lane);
  }
  struct Known { AttnTile x[ROWS / 32]; };
  __device__ __forceinline__ Known documents_of(int lane) const {
    Known known{};
    const int64_t t = (int64_t)(at + lane) * step + first;
    if (rows && t < end)
#pragma unroll
      for (int j = 0; j < ROWS / 32; ++j) known.x[j] = rows[t * (ROWS / 32) + j].documents;
    return known;
  }
  template <int N>
  static __device__ __forceinline__ Range keys_of(const AttnTile *tiles, int from, int to) {
    AttnTile x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = tiles[from / ATTN_TILE + i < to / ATTN_TILE ? from / ATTN_TILE + i : to / ATTN_TILE];
    Range r{INT32_MAX, -1, ATTN_ALL_PREFIX};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int all = r.flags & x[i].flags & ATTN_ALL_PREFIX;
      r = join(r, x[i]);
      r.flags = (r.flags & ~ATTN_ALL_PREFIX) | all | (x[i].flags & ATTN_SOME_PREFIX);
    }
    return r;
  }
  __device__ __forceinline__ void choose(const AttnCall &c, const Known &known, int lane) {
    const int64_t tt = (int64_t)(at + lane) * step + first;
    const bool there = tt < end;
    const int r0 = there ? (int)tt * ROWS : 0;
    const auto token = [&](int r) { return divide(c.by_group, r < c.rows ? r : c.rows - 1); };
    const int t0 = token(r0), t1 = token(r0 + ROWS - 1);
    const Range one = join(Range{INT32_MAX, -1, 0}, known.x[0]);
    const Range q = ROWS == 32 ? one : join(one, known.x[ROWS / 32 - 1]), mine_q = own == 0 ? one : join(Range{INT32_MAX, -1, 0}, known.x[ROWS / 32 - 1]);
    const Sight group = sees(c, t0 + c.offset, t1 + c.offset, q, group_from, group_to, group_docs);
    const Sight wave = sees(c, (ROWS == 32 ? t0 : token(r0 + own)) + c.offset, (ROWS == 32 ? t1 : token(r0 + own + 31)) + c.offset, mine_q, wave_from, wave_to, wave_docs);
    visit = __ballot(there && group.some);
    mine = __ballot(there && wave.some && r0 + own < c.rows);
    documents = __ballot(there && rows && !wave.documents);
    order = __ballot(there && !(wave.order && r0 + own + 32 <= c.rows));
    none = __ballot(there && rows && (q.flags & ATTN_SOME_NONE));
  }
  __device__ __forceinline__ Visit next(const AttnCall &c, int lane) {
    while (!visit) {
      if ((int64_t)(at + 64) * step + first >= end) return Visit{-1, false, false, false, false};
      at += 64;
      choose(c, documents_of(lane), lane);
    }
    const int i = __builtin_ctzll(visit);
    visit &= visit - 1;
    return Visit{(at + i) * step + first, (bool)((mine >> i) & 1), (bool)((documents >> i) & 1), (bool)((order >> i) & 1), (bool)((none >> i) & 1)};
  }
};

// A wavefront has 32 keys: their operands, and 2 x 32 x D sums, which with the scores fill half of a lane's registers (two wavefronts a SIMD) if the
// values stay in shared memory: they are read from there a block of 32 rows, as the queries and dy are.
//
// PARTS = 2: a workgroup has 64 keys and goes through 64 rows at a time, each wavefront through half of them.  Rows of 128 elements have no room for that.
template <class T, int D, int CAP, int SLOPE, int PARTS, int FINE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 64 && PARTS == 2 ? 3 : 2))) k_dkdv(const AttnCall c) {
#ifdef __HIP_DEVICE_COMPILE__
  constexpr int WAVES = 4, NT = 64 * WAVES, BLOCKS = WAVES / PARTS, KEYS = BLOCKS * 32, STEP = PARTS * 32, N = D / 32 / PARTS;
  typedef RowFeed<D, STEP, WAVES> Feed;
  typedef KeyFeed<D, KEYS, WAVES> Values;
  typedef __attribute__((address_space(3))) const AttnRows lds_rows;
  typedef __attribute__((address_space(3))) const f4 lds_f4;
  enum { ROWS = 2 * Feed::BYTES, STAGE = ROWS + PARTS * (int)sizeof(AttnRows), VALUES = 2 * STAGE, BYTES = VALUES + Values::BYTES };
  static_assert(sizeof(AttnRows) <= 1024, "a wavefront brings it in one load");
  constexpr int TURN = WAVES * turn_bytes(N), MEET = PARTS == 2 ? WAVES * N * 8192 : 0;
  __shared__ __attribute__((aligned(1024))) char shared[(int)BYTES > TURN + MEET ? (int)BYTES : TURN + MEET];
  __shared__ uint32_t words[WAVES][32];
  lds_char *lds = (lds_char *)shared, *values = lds + VALUES;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = wave / BLOCKS, block = wave % BLOCKS;
  const Place p = place_of(c, blockIdx.x, false);
  AttnShare share{p.tile, p.split, c.splits, p.tile * c.splits + p.split};
  if (c.shares) share = c.shares[(int64_t)p.b * c.share_slots + p.tile];
  if (share.tile < 0) return;
  const int key0 = share.tile * KEYS, wave_key = key0 + block * 32;
  const int h4 = (lane >> 5) * 4;
  s8 k[D / 16];
  uint32_t word = 0;
  {
    const int there = wave_key + (lane & 31) < c.keys ? wave_key + (lane & 31) : c.keys - 1;
    const uint16_t *kp = c.k.p + p.b * c.k.batch + there * c.k.token + p.h * c.k.head;
    if (c.k_words) word = c.k_words[(int64_t)p.b * c.tiles * ATTN_TILE + there];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const int d = i * 16 + (lane >> 5) * 8;
      k[i] = d < c.dim ? *(const s8 *)(kp + d) : s8{};
    }
    Values vf;
    vf.start(c.v, p.b, p.h, c.keys, c.dim, wave, lane);
    vf.load(key0, lds0 + VALUES, wave);
  }
  Feed qf, df;
  qf.start(c.q, p.b, p.h * c.group);
  df.start(c.dy, p.b, p.h * c.group);
  qf.keep(c, wave, lane);
  df.keep(c, wave, lane);
  const uint32_t *q_words = c.q_words ? c.q_words + (int64_t)p.b * c.q_tile_count * ATTN_TILE : nullptr;
  const AttnRows *row_data = c.row_data + (int64_t)p.hb * (c.rows_pad / 32);

  // without a prefix a causal mask leaves the rows from the first key's position on
  const int blocks = (c.rows + STEP - 1) / STEP;
  int first = 0;
  if (c.causal && !c.prefix && key0 > c.offset) {
    const int64_t f = (int64_t)(key0 - c.offset) * c.group / STEP;
    first = f < blocks ? (int)f : blocks;
  }
  RowWalk<KEYS, STEP> walk;
  walk.start(c, p, key0, wave_key, word, part * 32, first + share.part, share.parts, blocks, lane);
  if (lane < 32) words[wave][lane] = word;  // for this wavefront alone
  int lowered = 0;                          // of dk's sums and of ds
  f16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) dk[d] = dv[d] = f16{};

  const auto load = [&](int tile, int slot) {
    const uint32_t at = lds0 + slot * STAGE;
    qf.load(c, tile * STEP, at, wave, lane);
    df.load(c, tile * STEP, at + Feed::BYTES, wave, lane);
    if (wave < PARTS && lane < (int)sizeof(AttnRows) / 16)
      load_lds16(descriptor(row_data + tile * PARTS + wave, sizeof(AttnRows)), lane * 16, at + ROWS + wave * (int)sizeof(AttnRows));
  };
  int slot = 0;
  Visit next = walk.next(c, lane);
  if (next.tile >= 0) load(next.tile, 0);
  while (next.tile >= 0) {
    const Visit now = next;
    next = walk.next(c, lane);
    arrived();
    lds_char *queries = lds + slot * STAGE, *dys = queries + Feed::BYTES;
    lds_rows *known = (lds_rows *)(queries + ROWS) + part;
    if (now.some_none) {
      for (int idx = tid; idx < STEP * Shape<D>::CHUNKS; idx += NT) {
        const int i = idx / Shape<D>::CHUNKS, r = now.tile * STEP + i;
        if (r < c.rows && q_words[divide(c.by_group, r)] == ATTN_NONE) {
          clear_row<D>(queries, i, idx % Shape<D>::CHUNKS);
          clear_row<D>(dys, i, idx % Shape<D>::CHUNKS);
        }
      }
      arrived();
    }
    slot ^= 1;
    if (!now.run) {
      if (next.tile >= 0) load(next.tile, slot);
      continue;
    }
    f16 s = {}, dp = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = T::mfma(row_fragment<D>(queries, part * 32, i, lane), k[i], s);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) dp = T::mfma(row_fragment<D>(dys, part * 32, i, lane), row_fragment<D>(values, block * 32, i, lane), dp);
    __builtin_amdgcn_sched_barrier(0);      // reads of shared memory that are moved up from below would take the registers of k
    if (next.tile >= 0) load(next.tile, slot);
    const int rows_lowered = T::LIFT != 0 ? __builtin_amdgcn_readfirstlane(known->lowered) : 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f4 less = *(lds_f4 *)&known->less[g * 8 + h4];
      const f4 delta = *(lds_f4 *)&known->delta[g * 8 + h4];
      if (SLOPE) {
        const f4 slope2 = *(lds_f4 *)&known->slope2[g * 8 + h4];
        const i4 pos = *(__attribute__((address_space(3))) const i4 *)&known->pos[g * 8 + h4];
        const int key = wave_key + own_lane() % 32;
#pragma unroll
        for (int e = 0; e < 4; ++e) less[e] = fmaf(slope2[e], fabsf((float)(pos[e] - key)), less[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float weight, ds;
        gradient<CAP>(c, s[g * 4 + e], dp[g * 4 + e], less[e], delta[e], weight, ds);
        s[g * 4 + e] = weight;
        dp[g * 4 + e] = ds;
      }
    }
    if (now.masked()) {
      const int at = own_lane(), i = at & 31, row0 = now.tile * STEP + part * 32;
      const uint32_t mine = words[wave][i];
      uint32_t seen = now.documents ? same_words(mine & ~1u, known->word[i]) : ~0u;
      if (now.order) {
        // the rows from the key's own position on, as far as there are rows
        if (c.causal && !(mine & 1)) {
          const int position = wave_key + i - c.offset, first = (position > 0 ? position : 0) * c.group - row0;
          seen &= first > 31 ? 0u : ~0u << (first > 0 ? first : 0);
        }
        if (c.rows - row0 < 32) seen &= (1u << (c.rows - row0)) - 1;
      }
      seen >>= (at >> 5) * 4;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = where_seen(seen, r, s[r], 0);
        dp[r] = where_seen(seen, r, dp[r], 0);
      }
    }
    if (T::LIFT != 0 && (rows_lowered | lowered)) {      // some rows' ds are beyond float16
      if (rows_lowered > lowered) {
        take_down<D / 32>(dk, lowered - rows_lowered);
        lowered = rows_lowered;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = ldexpf(dp[r], -lowered);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const s8 pp = pack8<T>(s, i * 8), ds = pack8<T>(dp, i * 8);
      const s8 p_low = FINE ? pack8_low<T>(s, pp, i * 8) : s8{}, ds_low = FINE ? pack8_low<T>(dp, ds, i * 8) : s8{};
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        const s8 dy = column_fragment<D>(dys, part * 32 + i * 16, d, lane), query = column_fragment<D>(queries, part * 32 + i * 16, d, lane);
        dv[d] = T::mfma(dy, pp, dv[d]);
        dk[d] = T::mfma(query, ds, dk[d]);
        if (FINE) {
          dv[d] = T::mfma(dy, p_low, dv[d]);
          dk[d] = T::mfma(query, ds_low, dk[d]);
        }
      }
    }
  }
  arrived();                                // the values, where no block was visited; and nobody reads shared memory any more
  lds_char *own = lds + wave * turn_bytes(N);
  const int d0 = part * (N * 32);
  Argument *end = argument();
  const int width = end->width, keys = end->keys;
  const float scale = end->scale;
  const auto store = [&](const f16 (&k)[N], const f16 (&v)[N]) {
    if (share.parts > 1) {
      const int width4 = end->width4;
      const int64_t at = ((int64_t)p.hb * end->share_slots + share.slot) * KEYS + block * 32;
      const auto put = [&](float *out, int row, int d, f4 a, f4 b) {
        if (wave_key + row >= keys) return;
        out += (at + row) * width4 + d;
        if (d < width4) *(f4 *)out = a;
        if (d + 4 < width4) *(f4 *)(out + 4) = b;
      };
      float *part = end->part, *part2 = end->part2;
      by_rows(own, k, d0, lane, [&](int row, int d, f4 a, f4 b) { put(part, row, d, a, b); });
      by_rows(own, v, d0, lane, [&](int row, int d, f4 a, f4 b) { put(part2, row, d, a, b); });
      return;
    }
    const auto put = [&](uint16_t *out, int64_t token, int row, int d, f4 a, f4 b) {
      const int j = wave_key + row;
      if (j < keys) store8<T>(out + j * token, d, width, a, b);
    };
    uint16_t *dk = end->dk.p + p.b * end->dk.batch + p.h * end->dk.head, *dv = end->dv.p + p.b * end->dv.batch + p.h * end->dv.head;
    const int64_t dk_token = end->dk.token, dv_token = end->dv.token;
    by_rows(own, k, d0, lane, [&](int row, int d, f4 a, f4 b) { put(dk, dk_token, row, d, a, b); });
    by_rows(own, v, d0, lane, [&](int row, int d, f4 a, f4 b) { put(dv, dv_token, row, d, a, b); });
  };
  if constexpr (T::LIFT != 0) {
    take_down<D / 32>(dk, lowered - T::LIFT);
    take_down<D / 32>(dv, -T::LIFT);
  }
  if constexpr (PARTS == 2) {
    f16 sk[N], sv[N];
    lds_char *meet = lds + TURN;
    give<N>(meet + wave * (N * 8192), dk, sk, part == 1, lane);
    give<N>(meet + wave * (N * 8192) + N * 4096, dv, sv, part == 1, lane);
    __syncthreads();
    take<N>(meet + (wave ^ BLOCKS) * (N * 8192), sk, scale, scale, lane);
    take<N>(meet + (wave ^ BLOCKS) * (N * 8192) + N * 4096, sv, 1.f, 1.f, lane);
    store(sk, sv);
  } else {
#pragma unroll
    for (int d = 0; d < N; ++d) dk[d] *= scale;
    store(dk, dv);
  }
#endif
}

// ---------------------------------------------------------------------------------------------- launches
enum { FORWARD, FEW, DQ, DKDV };
template <class T, int WHAT, int D, int CAP, int SLOPE, int PARTS, int FINE>
bool launch(const AttnCall &c, const AttnLaunch &l) {
  hipStream_t st = (hipStream_t)l.stream;
  const dim3 grid(l.groups), block(256);
  if constexpr (WHAT == FORWARD) hipLaunchKernelGGL((k_forward<T, D, CAP, SLOPE, PARTS>), grid, block, 0, st, c);
  else if constexpr (WHAT == FEW) hipLaunchKernelGGL((k_forward_few<T, D, CAP, SLOPE>), grid, block, 0, st, c);
  else if constexpr (WHAT == DQ) hipLaunchKernelGGL((k_dq<T, D, CAP, SLOPE, PARTS, FINE>), grid, block, 0, st, c);
  else hipLaunchKernelGGL((k_dkdv<T, D, CAP, SLOPE, PARTS, FINE>), grid, block, 0, st, c);
  return hipGetLastError() == hipSuccess;
}
template <class T, int WHAT, int D, int CAP, int SLOPE>
bool launch_parts(const AttnCall &c, const AttnLaunch &l) {
  constexpr bool two = D == 64 ? WHAT != FEW : WHAT == FORWARD || WHAT == DQ, one = D == 128 || WHAT == DQ || WHAT == FEW;      // those that are chosen anywhere
  constexpr bool fine = WHAT == DQ || WHAT == DKDV;
  if constexpr (two) {
    if constexpr (fine)
      if (l.fine) return launch<T, WHAT, D, CAP, SLOPE, 2, 1>(c, l);
    if (!one || l.parts == 2) return launch<T, WHAT, D, CAP, SLOPE, 2, 0>(c, l);
  }
  if constexpr (one) {
    if constexpr (fine && !two)
      if (l.fine) return launch<T, WHAT, D, CAP, SLOPE, 1, 1>(c, l);
    return launch<T, WHAT, D, CAP, SLOPE, 1, 0>(c, l);
  }
  return false;
}
template <class T, int WHAT, int D>
bool launch_terms(const AttnCall &c, const AttnLaunch &l) {
  const bool cap = c.cap2 != 0.f, slope = c.slopes != nullptr;
  if (c.cap2 > 256 * 1.4427f) return launch_parts<T, WHAT, D, 2, 1>(c, l);      // 2^-23 of the cap is 2^-15; biased by nothing where there are no slopes
  if (cap) return slope ? launch_parts<T, WHAT, D, 1, 1>(c, l) : launch_parts<T, WHAT, D, 1, 0>(c, l);
  return slope ? launch_parts<T, WHAT, D, 0, 1>(c, l) : launch_parts<T, WHAT, D, 0, 0>(c, l);
}
template <class T, int WHAT>
bool launch_shape(const AttnCall &c, const AttnLaunch &l) {
  return l.dim == 64 ? launch_terms<T, WHAT, 64>(c, l) : launch_terms<T, WHAT, 128>(c, l);
}

}  // namespace chm_attention_kernels
#endif

// Attention: what its passes consist of, the small kernels around the tiles (documents, packing, joined sums), the entry points.
//
//   forward    [documents, packing] tiles [join]
//   backward   [packing] dq (and delta = dy.y), dk and dv [join]
// dq and dk with dv are kernels of their own, each of which works out the scores again: seven products in place of five, but no sums that several
// workgroups add to, so that the same inputs give the same bits.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/chm_measure.h"
#include "chm_attention.h"
#include "chm_elements.h"
#include "chm_strided.h"

namespace {

using namespace chm_elements;
typedef float f4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------- documents
struct DocumentsCall {
  const char *documents;                  // or null: all of one
  const uint8_t *prefix;                  // or null
  int64_t ld_documents, ld_prefix;
  uint32_t *words;
  AttnTile *tiles;
  int32_t n, index_bits, tiles_each;
};
// a wavefront for each tile of 64 tokens: those of the keys, behind them those of the queries
__device__ void documents_of(const DocumentsCall &a, const DocumentsCall &b, int64_t first, int64_t all, int64_t at_tile, int lane) {
  if (at_tile >= all) return;
  const bool second = at_tile >= first;
  const DocumentsCall &c = second ? b : a;
  const int block = (int)(at_tile - (second ? first : 0)), seq = block / c.tiles_each, tile = block - seq * c.tiles_each, t = tile * ATTN_TILE + lane;
  int64_t doc = -1;
  bool pre = false;
  if (t < c.n) {
    const int64_t at = seq * c.ld_documents + t;
    doc = !c.documents ? 0 : c.index_bits == 32 ? ((const int32_t *)c.documents)[at] : ((const int64_t *)c.documents)[at];
    pre = c.prefix && c.prefix[seq * c.ld_prefix + t] != 0;
  }
  const bool some = doc >= 0 && doc < INT32_MAX;
  const int64_t at = (int64_t)block * ATTN_TILE + lane;
  c.words[at] = some ? (uint32_t)doc * 2 + (pre ? 1 : 0) : ATTN_NONE;
  int lo = some ? (int)doc : INT32_MAX, hi = some ? (int)doc : -1;
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const int l = __shfl_xor(lo, d), h = __shfl_xor(hi, d);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
  }
  const uint64_t none = __ballot(!some && t < c.n), yes = __ballot(some && pre);      // places behind the last token are masked by their number
  if (lane == 0)
    c.tiles[block] = AttnTile{lo, hi, (none ? ATTN_SOME_NONE : 0) | (yes ? ATTN_SOME_PREFIX : 0) | (yes == ~0ull ? ATTN_ALL_PREFIX : 0), 0};
}

// ---------------------------------------------------------------------------------------------- packing
struct PackCall {
  struct { AttnInput in; uint16_t *out; int32_t tokens, heads; int64_t words; uint32_t groups; } m[4];
  int32_t count, dim, dim8;
};
// rows of dim elements one behind the other, rounded up to whole words of 8, zeros behind
__device__ void pack(const PackCall &c, uint32_t g) {
  int i = 0;
  while (i + 1 < c.count && g >= c.m[i].groups) g -= c.m[i++].groups;
  const auto &m = c.m[i];
  const int words = c.dim8 / 8;
  const int64_t w = (int64_t)g * 256 + threadIdx.x;
  if (w >= m.words) return;
  int64_t row = w / words;
  const int d = (int)(w - row * words) * 8;
  const int64_t token = row / m.heads;
  const int head = (int)(row - token * m.heads);
  const int64_t seq = token / m.tokens;
  const uint16_t *p = m.in.p + seq * m.in.batch + (token - seq * m.tokens) * m.in.token + head * m.in.head + d;
  Words v{0, 0, 0, 0};
  if (d + 8 <= c.dim) {
    v = load16((const char *)p);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (d + e < c.dim) v[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
  }
  *(Words *)(m.out + w * 8) = v;
}

// Both in one launch: neither waits for the other, and each is a few us (515 tokens, 6 heads of 72: 3 and 5)
__global__ void __launch_bounds__(256) k_prepare(DocumentsCall a, DocumentsCall b, int64_t first, int64_t all, uint32_t document_groups, PackCall c) {
  if (blockIdx.x < document_groups) documents_of(a, b, first, all, (int64_t)blockIdx.x * 4 + threadIdx.x / 64, threadIdx.x % 64);
  else pack(c, blockIdx.x - document_groups);
}

// ---------------------------------------------------------------------------------------------- joins
template <int DT>
__device__ __forceinline__ void put4(uint16_t *p, int d, int width, f4 v) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (d + e < width) Lane<DT>::put((char *)(p + d + e), v[e]);
}

// the parts of a row's softmax over the splits of its keys
template <int DT>
__global__ void __launch_bounds__(256) k_join_forward(const AttnCall c, int64_t all) {
  const int words = c.width4 / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= all) return;
  const int64_t at = i / words, rows = (int64_t)c.batch * c.kv_heads * c.rows;
  const int d = (int)(i - at * words) * 4;
  float top = c.part2[at * 2];
  for (int s = 1; s < c.splits; ++s) top = fmaxf(top, c.part2[(s * rows + at) * 2]);
  float sum = 0.f;
  f4 v{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < c.splits; ++s) {
    const float f = __builtin_amdgcn_exp2f(c.part2[(s * rows + at) * 2] - top);
    sum += c.part2[(s * rows + at) * 2 + 1] * f;
    v += *(const f4 *)(c.part + (s * rows + at) * c.width4 + d) * f;
  }
  const int64_t hb = at / c.rows, b = hb / c.kv_heads;
  const int h = (int)(hb - b * c.kv_heads), r = (int)(at - hb * c.rows), token = r / c.group, head = h * c.group + r - token * c.group;
  if (c.lse && d == 0) c.lse[hb * c.rows_pad + r] = sum == 0.f ? INFINITY : top + __builtin_amdgcn_logf(sum);
  v *= sum == 0.f ? 0.f : 1.f / sum;
  put4<DT>(c.y.p + b * c.y.batch + token * c.y.token + head * c.y.head, d, c.width, v);
  if (!c.low) return;
  f4 low;
#pragma unroll
  for (int e = 0; e < 4; ++e) low[e] = v[e] - (DT == CHM_BF16 ? bf16_up(bf16_down(v[e])) : f16_up(f16_down(v[e])));
  put4<DT>(c.low + ((b * c.tokens + token) * (c.kv_heads * c.group) + head) * c.width, d, c.width, low);
}

// dk and dv from the parts over the splits of the rows
template <int DT>
__global__ void __launch_bounds__(256) k_join_backward(const AttnCall c, int64_t all) {
  const int words = c.width4 / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= all) return;
  const int64_t at = i / words, hb = at / c.keys, b = hb / c.kv_heads, j = at - hb * c.keys;
  const int d = (int)(i - at * words) * 4, h = (int)(hb - b * c.kv_heads), tile = (int)(j / c.share_keys);
  AttnSlots slots{tile * c.splits, c.splits};
  if (c.shares) slots = c.tile_slots[b * c.share_tiles + tile];
  if (slots.count == 1) return;             // written as it was summed
  const int64_t step = (int64_t)c.share_keys * c.width4, from = (hb * c.share_slots + slots.first) * step + (j - (int64_t)tile * c.share_keys) * c.width4 + d;
  f4 k{0.f, 0.f, 0.f, 0.f}, v = k;
  for (int s = 0; s < slots.count; ++s) {
    k += *(const f4 *)(c.part + from + s * step);
    v += *(const f4 *)(c.part2 + from + s * step);
  }
  put4<DT>(c.dk.p + b * c.dk.batch + j * c.dk.token + h * c.dk.head, d, c.width, k);
  put4<DT>(c.dv.p + b * c.dv.batch + j * c.dv.token + h * c.dv.head, d, c.width, v);
}

// ---------------------------------------------------------------------------------------------- passes
int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }

AttnDivide divide_by(int64_t d) {
  if (d <= 1) return AttnDivide{0, 0};
  int l = 0;
  while ((1ll << l) < d) ++l;
  return AttnDivide{(uint32_t)((1ull << (31 + l)) / (uint64_t)d + 1), l - 1};
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

constexpr int FEW_ROWS = 32;
constexpr int64_t GROUPS_MAX = UINT32_MAX / 256;          // workgroups of a launch: threads are counted in 32 bits
constexpr int64_t LENGTH_MAX = 1ll << 30, ROWS_MAX = INT32_MAX - (1 << 13);

int64_t group_of(const chm_attention *a) { return a->heads / a->kv_heads; }
int64_t rows_pad(const chm_attention *a) { return up(a->tokens * group_of(a), ATTN_TILE) * ATTN_TILE; }
// Kept for the backward pass: lse of every row; what rounding took from y; what the documents of keys and queries are (laid out by sizes alone: the backward
// pass may name the same documents by other tensors)
uint64_t lse_bytes(const chm_attention *a) { return (uint64_t)(a->batch * a->kv_heads * rows_pad(a)) * 4; }
uint64_t low_bytes(const chm_attention *a) { return ((uint64_t)(a->batch * a->tokens * a->heads) * a->dim * 2 + 255) & ~255ull; }
// Without queries or without keys there is nothing to mask, and a tensor of no elements has no address
bool some_pairs(const chm_attention *a) { return a->batch > 0 && a->tokens > 0 && a->keys > 0; }
bool has_words(const chm_attention *a) { return some_pairs(a) && (a->k_documents || a->prefix); }
uint64_t documents_bytes(const chm_attention *a) {
  if (!has_words(a)) return 0;
  const int64_t tiles = a->batch * (up(a->keys, ATTN_TILE) + up(a->tokens, ATTN_TILE));
  return (uint64_t)tiles * (ATTN_TILE * 4 + sizeof(AttnTile)) + 4 * 256;
}
uint64_t saved_bytes(const chm_attention *a) { return lse_bytes(a) + low_bytes(a) + documents_bytes(a); }

// the strides of dimensions of one element say nothing
AttnInput input(const void *p, const int64_t s[3], int64_t b, int64_t t, int64_t h) {
  return AttnInput{(const uint16_t *)p, b > 1 ? s[0] : 0, t > 1 ? s[1] : 0, h > 1 ? s[2] : 0};
}
AttnOutput output(void *p, const int64_t s[3], int64_t b, int64_t t, int64_t h) {
  return AttnOutput{(uint16_t *)p, b > 1 ? s[0] : 0, t > 1 ? s[1] : 0, h > 1 ? s[2] : 0};
}

struct Pass {
  const chm_attention *a;
  Arena arena;
  hipStream_t st;
  bool run, ok = true;
  bool fits = true;                        // every launch's threads can be counted in 32 bits
  AttnCall c{};
  chm_attention_kernels chosen{0, 0, 0, 0, 0, 0, 1, 1, 0, 0};

  Pass(const chm_attention *a_, char *base, hipStream_t st_, bool run_) : a(a_), arena{base}, st(st_), run(run_) {
    const int64_t G = group_of(a), d8 = up(a->dim, 8) * 8;
    c.batch = (int32_t)a->batch;
    c.tokens = (int32_t)a->tokens;
    c.keys = (int32_t)a->keys;
    c.kv_heads = (int32_t)a->kv_heads;
    c.group = (int32_t)G;
    c.dim = (int32_t)d8;
    c.width = (int32_t)a->dim;
    c.width4 = (int32_t)up(a->dim, 4) * 4;
    c.rows = (int32_t)(a->tokens * G);
    c.rows_pad = (int32_t)rows_pad(a);
    c.offset = (int32_t)(a->keys - a->tokens);
    c.causal = a->causal != 0;
    c.tiles = (int32_t)up(a->keys, ATTN_TILE);
    c.q_tile_count = (int32_t)up(a->tokens, ATTN_TILE);
    c.by_group = divide_by(G);
    c.even_group = 32 % G == 0;
    const double log2e = 1.4426950408889634;
    c.scale = a->scale;
    c.to2 = (float)(a->scale * log2e);
    if (a->cap > 0) {
      c.tanh2 = (float)(2 * log2e * a->scale / a->cap);
      c.cap2 = (float)(a->cap * log2e);
      c.to_cap = (float)((double)a->scale / a->cap);
    }
    c.slopes = a->slopes;
    c.lse = (float *)a->saved;
    c.low = a->saved ? (uint16_t *)((char *)a->saved + lse_bytes(a)) : nullptr;
    c.prefix = a->prefix != nullptr;
    c.q = input(a->q, a->q_stride, a->batch, a->tokens, a->heads);
    c.k = input(a->k, a->k_stride, a->batch, a->keys, a->kv_heads);
    c.v = input(a->v, a->v_stride, a->batch, a->keys, a->kv_heads);
    chosen.dim = d8 <= 64 ? 64 : 128;
    c.heads_abreast = heads() % 8 == 0 ? 8 : (int32_t)heads();
    c.by_abreast = divide_by(c.heads_abreast);
    c.by_kv_heads = divide_by(a->kv_heads);
  }
  int64_t heads() const { return a->batch * a->kv_heads; }
  int64_t rows() const { return a->tokens * group_of(a); }
  bool bf16() const { return a->dtype == CHM_BF16; }

  uint32_t threads(int64_t groups, int64_t each) {
    fits = fits && groups <= UINT32_MAX / each;
    return (uint32_t)groups;
  }

  // a launch of `tiles` tiles of every head in `splits` parts
  AttnLaunch layout(int64_t tiles, int splits, int parts) {
    c.tiles_here = (int32_t)tiles;
    c.splits = splits;
    c.by_tiles = divide_by(tiles);
    c.by_splits = divide_by(splits);
    return AttnLaunch{chosen.dim, parts, chosen.fine, threads(heads() * tiles * splits, 256), st};
  }

  // Inputs as the tiles take them: 16-byte rows, and those of one load (`rows`) within offsets of 31 bits: what a load leaves out asks for an offset
  // just below 2^31 and arrives as zeros because no load's memory reaches that far
  PackCall pack{};
  void packed(AttnInput &in, int64_t tokens, int64_t heads, int64_t group, int rows, int bit) {
    const int64_t across = group == 1 ? rows - 1 : (rows - 1) / group + 1, most = ((1ll << 31) - 256) / 2 - 128;      // tokens, elements
    const bool reach = in.token <= most / across && (group == 1 || in.head <= (most - across * in.token) / (group - 1));
    if ((uintptr_t)in.p % 16 == 0 && a->dim % 8 == 0 && in.batch % 8 == 0 && in.token % 8 == 0 && in.head % 8 == 0 && reach) return;
    chosen.packed |= bit;
    const int64_t d8 = c.dim, words = a->batch * tokens * heads * (d8 / 8);
    auto &m = pack.m[pack.count++];
    m.in = in;
    m.out = (uint16_t *)arena.take((uint64_t)words * 16);
    m.tokens = (int32_t)tokens;
    m.heads = (int32_t)heads;
    m.words = words;
    m.groups = (uint32_t)up(words, 256);
    fits = fits && up(words, 256) < (1ll << 30);
    in = AttnInput{m.out, tokens * heads * d8, heads * d8, d8};
  }
  void inputs(const chm_attention_gradients *g) {
    packed(c.q, a->tokens, a->heads, group_of(a), 64, 1);
    packed(c.k, a->keys, a->kv_heads, 1, 64, 2);
    packed(c.v, a->keys, a->kv_heads, 1, g && dkdv_tile() == 128 ? 128 : 64, 4);      // dk and dv keep the values of all their keys
    if (g) packed(c.dy, a->tokens, a->heads, group_of(a), 64, 8);
    pack.dim = (int32_t)a->dim;
    pack.dim8 = c.dim;
    int64_t packs = 0, first = 0, all = 0;
    for (int i = 0; i < pack.count; ++i) packs += pack.m[i].groups;
    DocumentsCall kd{(const char *)a->k_documents, a->prefix, a->ld_k_documents, a->ld_prefix, nullptr, nullptr, c.keys, a->index_bits, c.tiles};
    DocumentsCall qd{(const char *)a->q_documents, nullptr, a->ld_q_documents, 0, nullptr, nullptr, c.tokens, a->index_bits, c.q_tile_count};
    if (has_words(a)) {
      Arena kept{a->saved ? (char *)a->saved + lse_bytes(a) + low_bytes(a) : nullptr};      // written by the forward pass, if there is one to come back to
      const bool keep = g || a->saved;
      Arena &from = keep ? kept : arena;
      const auto room = [&](DocumentsCall &d) {
        d.words = (uint32_t *)from.take((uint64_t)a->batch * d.tiles_each * ATTN_TILE * 4);
        d.tiles = (AttnTile *)from.take((uint64_t)a->batch * d.tiles_each * sizeof(AttnTile));
      };
      room(kd);
      // the queries' tokens are the keys': their words are (the prefix is asked of keys alone)
      const bool same = !keep && a->tokens == a->keys && a->q_documents == a->k_documents && (a->batch == 1 || a->ld_q_documents == a->ld_k_documents);
      if (same) qd.words = kd.words, qd.tiles = kd.tiles;
      else room(qd);
      c.k_words = kd.words; c.k_tiles = kd.tiles;
      c.q_words = qd.words; c.q_tiles = qd.tiles;
      if (!run) c.k_words = c.q_words = (const uint32_t *)1;      // only whether there are any is asked
      first = a->batch * kd.tiles_each;
      all = g ? 0 : first + (same ? 0 : a->batch * qd.tiles_each);
    }
    const int64_t documents = up(all, 4);
    const uint32_t n = threads(documents + packs, 256);
    if (run && fits && n) {
      hipLaunchKernelGGL(k_prepare, dim3(n), dim3(256), 0, st, kd, qd, first, all, (uint32_t)documents, pack);
      ok = ok && hipGetLastError() == hipSuccess;
    }
  }

  // Parts of the keys of the kernel for few rows: as many workgroups as run at once (1 a compute unit, 2 with rows of 64), in whole rounds.  us by parts, 32
  // heads of 128, 8 of keys: 8 answers of 32,768 keys 426 (1), 237 (2), 181 (4), 179 (8); one of 65,536 629 (1), 177 (4), 92 (8), 47 (32); 4 of 4,096 46 (1), 18 (4), 16
  // (8); 64 answers of 2,048 keys, 16 heads of 64 104 (1), 106 (2), 128 (8).
  static int few_splits(int64_t heads, int64_t tiles, int dim) {
    const int64_t slots = dim == 64 ? 512 : 256;
    int best = 1;
    double least = 1e30;
    for (int64_t s = 1; s <= 64 && (s == 1 || (s * 4 <= tiles && heads * s <= GROUPS_MAX)); ++s) {
      const double cost = (double)up(heads * s, slots) / s + 0.002 * s;
      if (cost < least) least = cost, best = (int)s;
    }
    return best;
  }
  // Parts of the sums of a tile kernel with `groups` workgroups, each of which goes through `steps` of 64: as many as fill `slots`, of `least` steps and more
  // (forward, 512 workgroups run at once, three a compute unit with rows of 64: 768)
  static int tile_splits(int64_t groups, int64_t steps, int64_t slots, int64_t least) {
    int64_t s = slots / (groups < 1 ? 1 : groups);
    if (s > steps / least) s = steps / least;
    return (int)(s < 1 ? 1 : s < 16 ? s : 16);
  }
  // Of dk and dv, equal ones: as many as run at once, two a compute unit; with a causal mask, where the first keys see the most rows, twice as many if each
  // keeps work enough to be worth its sums' way through memory in float32 (32 heads, 8 of keys, 128; us with the join, by parts: 2,048 tokens without a mask 455
  // (1), 169 (4), 198 (8); 8,192 tokens causal 2,087 (1), 1,297 (2), 1,308 (4)).  Rows of 64 have twice the workgroups and half the steps: 16 heads, 512 tokens 15
  // (1), 18 (2).
  static int dkdv_splits(int64_t groups, int64_t steps, bool causal, int dim) {
    const int a = tile_splits(groups, steps, 512, dim == 64 ? 8 : 4), b = causal ? tile_splits(groups, steps, 1024, 16) : 1;
    return a > b ? a : b;
  }
  // Where a mask makes the tiles of keys differ, their parts are shared out on the GPU by what they cost, and the longest run first: as many as 1,024 workgroups, and
  // with documents the order alone where there are more.  us against equal parts, both with the join, 32 heads, 8 of keys, 128: 4,096 packed tokens 129 and
  // 150; causal 1,024 tokens 51 and 55, 2,048 tokens 109 and 126, 4 x 1,024 tokens 130 and 151, 4,096 tokens 360 and 353; 8,192 tokens (512 tiles) 1,390 and 1,350.
  int dealt_parts() const { return tile_splits(heads() * key_tiles(), up(rows(), ATTN_TILE), 1024, chosen.dim == 64 ? 16 : 2); }
  bool dealt() const {
    const int64_t groups = heads() * key_tiles();
    if (a->tokens == 0 || a->keys == 0 || key_tiles() > ATTN_SHARE_TILES || c.q_tile_count > ATTN_SHARE_QUERIES) return false;
    return a->k_documents ? dealt_parts() > 1 || groups > 512 : a->causal && groups < 512 && dealt_parts() > 1;
  }
  int dkdv_tile() const { return chosen.dim == 64 ? 64 : 128; }
  int64_t key_tiles() const { return up(a->keys, dkdv_tile()); }

  // Rows of a workgroup.  64 of them take half as long as 128 but read the keys twice as often: taken where the whole launch is no more than the workgroups
  // that run at once, with a causal mask, where they differ, twice that.  Rows of 64 elements leave room for a third workgroup with 64 rows, and only dq in large
  // calls is the better for 128.  us with 64 and 128 rows, 32 heads, 8 of keys, 128, causal, forward and dq: 512 tokens 18 + 21 and 23 + 29, 2,048 tokens 65 + 77 and 71 + 90,
  // without a mask 106 + 125 and 87 + 114, 4,096 tokens 212 + 258 and 175 + 230; 256 tokens over 2,048 keys 31 and 33 with the join, over 8,192 58 and 55.  64: 4 x 2,048
  // tokens of 16 heads 72 + 92 and 85 + 102, 8,000 of 32 heads 413 + 532 and 418 + 488.
  bool few_groups() const { return heads() * up(rows(), 128) <= (a->causal ? 512 : 256); }
  int forward_tile() const { return chosen.dim == 64 || (few_groups() && c.tiles < 64) ? 64 : 128; }
  int dq_tile() const { return chosen.dim == 64 ? (heads() * up(rows(), 128) <= 1024 ? 64 : 128) : few_groups() ? 64 : 128; }

  void forward(void *y, const int64_t y_stride[3]) {
    c.y = output(y, y_stride, a->batch, a->tokens, a->heads);
    if (a->batch == 0 || a->tokens == 0) return;
    inputs(nullptr);
    chosen.few = rows() <= FEW_ROWS;
    const int64_t all = heads() * rows(), joins = up(all * (c.width4 / 4), 256);
    AttnLaunch l;
    if (chosen.few) {
      chosen.forward_rows = FEW_ROWS;
      l = layout(1, joins <= GROUPS_MAX ? few_splits(heads(), c.tiles, chosen.dim) : 1, 1);
    } else {
      chosen.forward_rows = forward_tile();
      const int64_t tiles = up(rows(), chosen.forward_rows);
      l = layout(tiles, tile_splits(heads() * tiles, c.tiles, chosen.dim == 64 ? 768 : 512, 8), 128 / chosen.forward_rows);
    }
    chosen.forward_splits = c.splits;
    if (c.splits > 1) {
      c.part = (float *)arena.take((uint64_t)(c.splits * all * c.width4) * 4);
      c.part2 = (float *)arena.take((uint64_t)(c.splits * all * 2) * 4);
      threads(joins, 256);
    }
    if (!run || !fits) return;
    ok = ok && (bf16() ? attn_forward_bf16 : attn_forward_f16)(c, l, chosen.few);
    if (c.splits > 1) {
      if (bf16()) hipLaunchKernelGGL(k_join_forward<CHM_BF16>, dim3((uint32_t)joins), dim3(256), 0, st, c, all * (c.width4 / 4));
      else hipLaunchKernelGGL(k_join_forward<CHM_F16>, dim3((uint32_t)joins), dim3(256), 0, st, c, all * (c.width4 / 4));
      ok = ok && hipGetLastError() == hipSuccess;
    }
  }

  void backward(const chm_attention_gradients *g) {
    if (a->batch == 0) return;
    const int64_t B = a->batch, T = a->tokens, K = a->keys;
    c.dy = input(g->dy, g->dy_stride, B, T, a->heads);
    c.y_in = input(g->y, g->y_stride, B, T, a->heads);
    c.dq = output(g->dq, g->dq_stride, B, T, a->heads);
    c.dk = output(g->dk, g->dk_stride, B, K, a->kv_heads);
    c.dv = output(g->dv, g->dv_stride, B, K, a->kv_heads);
    inputs(g);
    chosen.fine = heads() * up(rows(), 64) <= 128;      // then dq's workgroups have 64 rows, one for every other compute unit at most
    c.row_data = (AttnRows *)arena.take((uint64_t)(heads() * c.rows_pad / 32) * sizeof(AttnRows));
    chosen.dkdv_keys = dkdv_tile();
    const int64_t tiles = key_tiles();
    const bool shared = dealt();
    const int splits = shared ? dealt_parts() : dkdv_splits(heads() * tiles, up(rows(), ATTN_TILE), a->causal != 0, chosen.dim);
    c.share_tiles = (int32_t)tiles;
    c.share_keys = chosen.dkdv_keys;
    c.share_slots = (int32_t)(tiles * splits);
    c.share_unit = (int32_t)(chosen.dim == 64 ? group_of(a) : 2 * group_of(a));
    c.share_least = 4;
    c.share_short = chosen.dim == 64 ? 8 : 64;
    if (T > 0) {
      chosen.dq_rows = dq_tile();
      AttnLaunch l = layout(up(rows(), chosen.dq_rows), 1, 128 / chosen.dq_rows);
      if (shared) {                        // worked out beside dq
        c.shares = (AttnShare *)arena.take((uint64_t)(a->batch * c.share_slots) * sizeof(AttnShare));
        c.tile_slots = (AttnSlots *)arena.take((uint64_t)(a->batch * c.share_tiles) * sizeof(AttnSlots));
        c.share_groups = (int32_t)a->batch;
        l.groups = threads((int64_t)l.groups + a->batch, 256);
      }
      if (run && fits) ok = ok && (bf16() ? attn_dq_bf16 : attn_dq_f16)(c, l);
    }
    if (K > 0) {
      const AttnLaunch l = shared ? layout(c.share_slots, 1, 128 / chosen.dkdv_keys) : layout(tiles, splits, 128 / chosen.dkdv_keys);
      chosen.dkdv_splits = splits;
      chosen.dkdv_shared = shared;
      const int64_t words = heads() * K * (c.width4 / 4), joins = up(words, 256);
      if (splits > 1) {
        const uint64_t bytes = (uint64_t)(heads() * c.share_slots) * (uint64_t)(chosen.dkdv_keys * c.width4) * 4;
        c.part = (float *)arena.take(bytes);
        c.part2 = (float *)arena.take(bytes);
        threads(joins, 256);
      }
      if (!run || !fits) return;
      ok = ok && (bf16() ? attn_dkdv_bf16 : attn_dkdv_f16)(c, l);
      if (splits > 1) {
        if (bf16()) hipLaunchKernelGGL(k_join_backward<CHM_BF16>, dim3((uint32_t)joins), dim3(256), 0, st, c, words);
        else hipLaunchKernelGGL(k_join_backward<CHM_F16>, dim3((uint32_t)joins), dim3(256), 0, st, c, words);
        ok = ok && hipGetLastError() == hipSuccess;
      }
    }
  }
};

bool aligned(const void *p, int64_t to) { return (uintptr_t)p % to == 0; }
using chm_strided::countable;
bool fine(const int64_t s[3], int64_t b, int64_t t, int64_t h) { return countable(s[0], b) && countable(s[1], t) && countable(s[2], h); }

int check(const chm_attention *a) {
  if (!a || (a->dtype != CHM_BF16 && a->dtype != CHM_F16)) return CHM_ERR_ARG;
  if (a->batch < 0 || a->batch > INT32_MAX || a->tokens < 0 || a->tokens > LENGTH_MAX || a->keys < 0 || a->keys > LENGTH_MAX) return CHM_ERR_ARG;
  if (a->kv_heads < 1 || a->kv_heads > (1 << 20) || a->heads < a->kv_heads || a->heads > (1 << 20) || a->heads % a->kv_heads || a->dim < 1 || a->dim > 128) return CHM_ERR_ARG;
  if (a->tokens * group_of(a) > ROWS_MAX || a->batch * a->kv_heads > INT32_MAX) return CHM_ERR_ARG;
  if (a->batch * a->kv_heads > 0 && rows_pad(a) > (1ll << 50) / (a->batch * a->kv_heads)) return CHM_ERR_ARG;
  if (!(a->scale > 0) || !(a->cap >= 0) || !isfinite(a->cap)) return CHM_ERR_ARG;
  if (a->scale > 1e30f || (a->cap > 0 && a->scale / a->cap > 1e30f)) return CHM_ERR_ARG;       // what products are multiplied by has to be finite
  if (!fine(a->q_stride, a->batch, a->tokens, a->heads) || !fine(a->k_stride, a->batch, a->keys, a->kv_heads) ||
      !fine(a->v_stride, a->batch, a->keys, a->kv_heads)) return CHM_ERR_ARG;
  if (!aligned(a->q, 2) || !aligned(a->k, 2) || !aligned(a->v, 2) || !aligned(a->saved, 16) || !aligned(a->slopes, 4)) return CHM_ERR_ARG;
  if ((some_pairs(a) && !a->q_documents != !a->k_documents) || (a->prefix && !a->causal)) return CHM_ERR_ARG;
  if (a->q_documents || a->k_documents) {
    if (a->index_bits != 32 && a->index_bits != 64) return CHM_ERR_ARG;
    if (!aligned(a->q_documents, a->index_bits / 8) || !aligned(a->k_documents, a->index_bits / 8)) return CHM_ERR_ARG;
    if (a->batch > 1 && (!countable(a->ld_q_documents, a->batch) || !countable(a->ld_k_documents, a->batch))) return CHM_ERR_ARG;
  }
  if (a->prefix && a->batch > 1 && !countable(a->ld_prefix, a->batch)) return CHM_ERR_ARG;
  return CHM_OK;
}

int check_gradients(const chm_attention *a, const chm_attention_gradients *g) {
  if (!g || !fine(g->dy_stride, a->batch, a->tokens, a->heads) || !fine(g->y_stride, a->batch, a->tokens, a->heads) ||
      !fine(g->dq_stride, a->batch, a->tokens, a->heads) || !fine(g->dk_stride, a->batch, a->keys, a->kv_heads) ||
      !fine(g->dv_stride, a->batch, a->keys, a->kv_heads)) return CHM_ERR_ARG;
  if (!aligned(g->dy, 2) || !aligned(g->y, 2) || !aligned(g->dq, 2) || !aligned(g->dk, 2) || !aligned(g->dv, 2)) return CHM_ERR_ARG;
  return CHM_OK;
}

using chm_strided::Dim;
using chm_strided::Tensor;
Tensor tensor(const chm_attention *a, const void *p, const int64_t s[3], int64_t tokens, int64_t heads) {
  return Tensor(p, a->dim, 2, {Dim{a->batch, s[0]}, Dim{tokens, s[1]}, Dim{heads, s[2]}});
}
Tensor bytes(const void *p, uint64_t n) { return Tensor(p, (int64_t)n, 1, {Dim{1, 0}, Dim{1, 0}, Dim{1, 0}}); }
Tensor rows(const void *p, int64_t n, int64_t width, int64_t ld, int size) { return Tensor(p, width, size, {Dim{n, ld}, Dim{1, 0}, Dim{1, 0}}); }

// whether one of the results lies over another one, over itself, or over an input
template <int R, int I>
bool clash(const Tensor (&results)[R], const Tensor (&inputs)[I]) {
  for (int r = 0; r < R; ++r) {
    if (!results[r].apart()) return true;
    for (int i = 0; i < I; ++i)
      if (chm_strided::share(results[r], inputs[i])) return true;
    for (int o = 0; o < r; ++o)
      if (chm_strided::share(results[r], results[o])) return true;
  }
  return false;
}

bool clash_forward(const chm_attention *a, void *y, const int64_t s[3], void *scratch, uint64_t scratch_bytes) {
  const Tensor results[] = {tensor(a, y, s, a->tokens, a->heads), bytes(a->saved, a->saved ? saved_bytes(a) : 0), bytes(scratch, scratch_bytes)};
  const Tensor inputs[] = {tensor(a, a->q, a->q_stride, a->tokens, a->heads), tensor(a, a->k, a->k_stride, a->keys, a->kv_heads),
                           tensor(a, a->v, a->v_stride, a->keys, a->kv_heads), bytes(a->slopes, a->slopes ? a->heads * 4 : 0),
                           rows(a->q_documents, a->batch, a->tokens, a->ld_q_documents, a->index_bits / 8),
                           rows(a->k_documents, a->batch, a->keys, a->ld_k_documents, a->index_bits / 8), rows(a->prefix, a->batch, a->keys, a->ld_prefix, 1)};
  return clash(results, inputs);
}

bool clash_backward(const chm_attention *a, const chm_attention_gradients *g, void *scratch, uint64_t scratch_bytes) {
  const Tensor results[] = {tensor(a, g->dq, g->dq_stride, a->tokens, a->heads), tensor(a, g->dk, g->dk_stride, a->keys, a->kv_heads),
                            tensor(a, g->dv, g->dv_stride, a->keys, a->kv_heads), bytes(scratch, scratch_bytes)};
  const Tensor inputs[] = {tensor(a, a->q, a->q_stride, a->tokens, a->heads), tensor(a, a->k, a->k_stride, a->keys, a->kv_heads),
                           tensor(a, a->v, a->v_stride, a->keys, a->kv_heads), tensor(a, g->dy, g->dy_stride, a->tokens, a->heads),
                           tensor(a, g->y, g->y_stride, a->tokens, a->heads), bytes(a->saved, saved_bytes(a)), bytes(a->slopes, a->slopes ? a->heads * 4 : 0),
                           rows(a->q_documents, a->batch, a->tokens, a->ld_q_documents, a->index_bits / 8),
                           rows(a->k_documents, a->batch, a->keys, a->ld_k_documents, a->index_bits / 8), rows(a->prefix, a->batch, a->keys, a->ld_prefix, 1)};
  return clash(results, inputs);
}

const int64_t ANY[3] = {0, 0, 0};

}  // namespace

extern "C" int chm_attention_sizes(const chm_attention *a, const chm_attention_gradients *g, uint64_t *saved, uint64_t *forward_scratch, uint64_t *backward_scratch) {
  const int rc = check(a);
  if (rc != CHM_OK) return rc;
  if (g && check_gradients(a, g) != CHM_OK) return CHM_ERR_ARG;
  if (saved) *saved = saved_bytes(a);
  if (forward_scratch) {
    Pass p(a, nullptr, nullptr, false);
    p.forward(nullptr, ANY);
    if (!p.fits) return CHM_ERR_ARG;
    *forward_scratch = p.arena.used;
  }
  if (backward_scratch) {
    *backward_scratch = 0;
    if (!g) return CHM_OK;
    Pass p(a, nullptr, nullptr, false);
    p.backward(g);
    if (!p.fits) return CHM_ERR_ARG;
    *backward_scratch = p.arena.used;
  }
  return CHM_OK;
}

extern "C" int chm_attention_selection(const chm_attention *a, const chm_attention_gradients *g, chm_attention_kernels *out) {
  if (!out || check(a) != CHM_OK || (g && check_gradients(a, g) != CHM_OK)) return CHM_ERR_ARG;
  Pass p(a, nullptr, nullptr, false);
  p.forward(nullptr, ANY);
  if (!p.fits) return CHM_ERR_ARG;
  *out = p.chosen;
  if (g) {
    Pass b(a, nullptr, nullptr, false);
    b.backward(g);
    if (!b.fits) return CHM_ERR_ARG;
    out->packed = b.chosen.packed;
    out->dq_rows = b.chosen.dq_rows;
    out->dkdv_keys = b.chosen.dkdv_keys;
    out->dkdv_splits = b.chosen.dkdv_splits;
    out->dkdv_shared = b.chosen.dkdv_shared;
    out->fine = b.chosen.fine;
  }
  return CHM_OK;
}

extern "C" int chm_attention_forward(const chm_attention *a, void *y, const int64_t y_stride[3], void *scratch, uint64_t scratch_bytes, void *hip_stream) {
  const int rc = check(a);
  if (rc != CHM_OK) return rc;
  if (!y_stride || !fine(y_stride, a->batch, a->tokens, a->heads) || !aligned(y, 2) || !aligned(scratch, 16)) return CHM_ERR_ARG;
  if (a->batch == 0 || a->tokens == 0) return CHM_OK;
  if (!a->q || !y || (a->keys > 0 && (!a->k || !a->v))) return CHM_ERR_ARG;
  Pass need(a, nullptr, nullptr, false);
  need.forward(y, y_stride);
  if (!need.fits) return CHM_ERR_ARG;
  if (need.arena.used && !scratch) return CHM_ERR_ARG;
  if (scratch_bytes < need.arena.used) return CHM_ERR_LIMIT;
  if (clash_forward(a, y, y_stride, scratch, need.arena.used)) return CHM_ERR_ARG;
  Pass p(a, (char *)scratch, (hipStream_t)hip_stream, true);
  p.forward(y, y_stride);
  return p.ok ? CHM_OK : CHM_ERR_HIP;
}

extern "C" int chm_attention_backward(const chm_attention *a, const chm_attention_gradients *g, void *scratch, uint64_t scratch_bytes, void *hip_stream) {
  int rc = check(a);
  if (rc == CHM_OK) rc = check_gradients(a, g);
  if (rc != CHM_OK) return rc;
  if (!aligned(scratch, 16)) return CHM_ERR_ARG;
  if (a->batch == 0 || (a->tokens == 0 && a->keys == 0)) return CHM_OK;
  if (a->tokens > 0 && (!a->q || !g->dy || !g->y || !g->dq || !a->saved)) return CHM_ERR_ARG;
  if (a->keys > 0 && (!a->k || !a->v || !g->dk || !g->dv)) return CHM_ERR_ARG;
  Pass need(a, nullptr, nullptr, false);
  need.backward(g);
  if (!need.fits) return CHM_ERR_ARG;
  if (need.arena.used && !scratch) return CHM_ERR_ARG;
  if (scratch_bytes < need.arena.used) return CHM_ERR_LIMIT;
  if (clash_backward(a, g, scratch, need.arena.used)) return CHM_ERR_ARG;
  Pass p(a, (char *)scratch, (hipStream_t)hip_stream, true);
  p.backward(g);
  return p.ok ? CHM_OK : CHM_ERR_HIP;
}

// Attention: what its host part (chm_attention.hip) hands to its kernels (chm_attention_kernels.h).  Internal to libchm.
//
// The query heads that share a key head (a group of G) are rows of one matrix: row r of (sequence, key head) is token r / G, head r % G of the
// group.  A lane knows its row's token and slope, so nothing else changes, keys and values are read once a group, and a single token's heads fill the
// rows of a matrix instruction.
#ifndef CHM_ATTENTION_H
#define CHM_ATTENTION_H
#include <stdint.h>

#include "../../include/chm_operators.h"

// Elements of 16 bits; strides in elements.  Inputs: every row of `dim` starts on 16 bytes and dim is a multiple of 8 (others are packed first).
struct AttnInput { const uint16_t *p; int64_t batch, token, head; };
struct AttnOutput { uint16_t *p; int64_t batch, token, head; };

// r / d for r below 2^31: the upper half of r m, shifted; d = 1: m = 0
struct AttnDivide { uint32_t m; int32_t shift; };

// What 64 tokens' documents are: the least and the largest number (first > last: none), and flags.  A document and "in the prefix" of a token
// are one word: number * 2 + prefix (the largest is 0xfffffffd).
struct AttnTile { int32_t first, last, flags, unused; };
enum { ATTN_SOME_NONE = 1, ATTN_SOME_PREFIX = 2, ATTN_ALL_PREFIX = 4 };
constexpr uint32_t ATTN_NONE = 0xfffffffeu;
constexpr int ATTN_TILE = 64;              // keys of a tile; words and tiles are laid out for whole ones

// What the kernel of dq leaves to that of dk and dv about 32 rows, one value after the other (rows behind the last see nothing)
struct AttnRows {
  float less[32];                          // log2 of the sum of powers of two, less cap2 where there is a cap up to 256, less the lift of p; +inf: the row sees nothing
  float delta[32];                         // dy . y; with a cap four times that
  uint32_t word[32];                       // document * 2; ATTN_NOBODY: none
  float slope2[32];
  int32_t pos[32];
  AttnTile documents;                      // of all of them
  int32_t lowered, unused[3];              // float16: ds is within its range if lifted by so much less
};
constexpr uint32_t ATTN_NOBODY = 0xffffffffu;      // odd: equal to no key's word without its lowest bit, ATTN_NONE among them

// A workgroup of dk and dv: its tile of keys (-1: none), the parts that the rows are dealt to and which of them it is, and where its sums go if there are several
struct AttnShare { int32_t tile, part, parts, slot; };
struct AttnSlots { int32_t first, count; };

struct AttnCall {
  AttnInput q, k, v, dy;
  AttnInput y_in;                          // the forward pass's result, at any alignment
  AttnOutput y, dq, dk, dv;
  int32_t batch, tokens, keys, kv_heads, group, dim, width;      // dim: elements of the inputs' rows; width: of the outputs' (dim less what packing added)
  int32_t rows, rows_pad;                  // tokens * group, rounded up to whole tiles
  int32_t offset;                          // keys - tokens: position of the first query
  int32_t causal, tiles;                   // tiles of 64 keys
  AttnDivide by_group;
  int32_t even_group;                      // 32 is a multiple of the group
  float scale;                             // of the gradients dq and dk
  float to2;                               // score in powers of two: scale * log2(e)
  float tanh2, cap2, to_cap;               // 2 scale / cap * log2(e); cap * log2(e); scale / cap
  const float *slopes;                     // [kv_heads * group], or null
  const uint32_t *q_words, *k_words;       // [batch][whole tiles], or null: no documents and no prefix
  const AttnTile *q_tiles, *k_tiles;       // [batch][tiles]
  int32_t q_tile_count;
  int32_t prefix;                          // some words may have the prefix's bit
  float *lse;                              // [batch * kv_heads][rows_pad]: kept by the forward pass
  uint16_t *low;                           // [batch, tokens, heads, width]: what rounding took from y
  AttnRows *row_data;                      // [batch * kv_heads][rows_pad / 32]
  // sums split over workgroups: float32 parts, joined in order
  int32_t splits;
  float *part, *part2;                     // forward: [splits][batch * kv_heads][rows][width4] and (maximum, sum); backward: dk and dv [batch * kv_heads][share_slots][keys of a tile][width4]
  int32_t width4;                          // width rounded up to 4
  // layout of the launch: the workgroups' tiles of rows or keys
  int32_t tiles_here, heads_abreast;
  AttnDivide by_abreast, by_splits, by_tiles, by_kv_heads;
  // dk and dv: `share_slots` parts of the sums of a sequence's tiles of keys (share_keys each).  Shared out by the first workgroups of dq's launch, or (null) evenly:
  // `splits` for each tile
  AttnShare *shares;                       // [batch][share_slots]
  AttnSlots *tile_slots;                   // [batch][share_tiles]
  int32_t share_groups, share_tiles, share_keys, share_slots;
  int32_t share_unit, share_least, share_short;            // blocks of rows of 64 tokens; fewest blocks of a part; most of one that is short
};

enum { ATTN_SHARE_TILES = 1024, ATTN_SHARE_QUERIES = 1024 };        // most tiles of keys and of queries that are shared out on the GPU
// Kernels of a pass; dim: 64 or 128; parts: wavefronts that share a sum, 1 or 2; fine: gradients by twice the products.  false: HIP failed.
struct AttnLaunch { int32_t dim, parts, fine; uint32_t groups; void *stream; };
bool attn_forward_bf16(const AttnCall &c, const AttnLaunch &l, bool few);
bool attn_forward_f16(const AttnCall &c, const AttnLaunch &l, bool few);
bool attn_dq_bf16(const AttnCall &c, const AttnLaunch &l);
bool attn_dq_f16(const AttnCall &c, const AttnLaunch &l);
bool attn_dkdv_bf16(const AttnCall &c, const AttnLaunch &l);
bool attn_dkdv_f16(const AttnCall &c, const AttnLaunch &l);
#endif

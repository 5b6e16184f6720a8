// Layout of one matrix product of the gated feed-forward block and the launch interface between its host part
// (chm_ffn.hip) and its tile kernels (chm_gemm.h).  Internal to libchm.
#ifndef CHM_FFN_H
#define CHM_FFN_H
#include <stdint.h>

#include "../../include/chm_operators.h"

// An operand of C[m, n] = sum_k A[m, k] B[n, k]: its base (two bases: two weights side by side, or two runs of k one behind the
// other), elements from one row of memory to the next, length of a run of k.  Elements of 16 bits, 16-byte aligned rows.
struct GemmOperand { const void *p[2]; int64_t ld, k; };

// The projections g and u as the backward pass reads them: blocks of 16 rows x 32 features, `blocks` of them side by side (layout: chm_gemm.h)
struct Kept { char *p; int64_t blocks; };

struct GemmCall {
  GemmOperand a, b;
  int64_t m, n;                 // sizes of the product (n: features of one weight in a two-weight product)
  int32_t tiles_m, tiles_n;
  int32_t runs;                 // 2: a second run of k follows the first, from the operands' second bases
  int32_t splits;               // > 1: the sums are split over workgroups, float32 parts go to `part`
  int32_t act;
  // plain store: c[0] for rows below m_first, c[1] (row m - m_first) from there on; rows up to m_real, columns up to n_real
  void *c[2];
  int64_t ldc;
  int64_t m_first, m_real, n_real;
  int32_t f32_out, accumulate;
  float *part;                  // [splits][m][ld_part]
  int64_t ld_part;              // columns rounded up to 8
  // two-weight product and gradient of the activation: internal buffers of `ldi` elements a row
  uint16_t *h;
  Kept kept;                    // null: not kept
  uint16_t *dgate, *dup;
  int64_t ldi, ldd;             // ldd: row of dgate / dup
};

// Products that one launch works out.  GEMM_BACK: dx (the longest sums, first), then both weight gradients, which depend on nothing but what
// GEMM_DH has left: together they fill the compute units that each alone leaves idle at its end.
enum { GEMM_GATE_UP = 0, GEMM_OUT = 1, GEMM_DH = 2, GEMM_BACK = 3 };
struct GemmGroup {
  GemmCall call[3];
  int32_t count;
  int32_t first[4];             // first workgroup of each call (a multiple of 8), and one behind the last
};

// Tiles of 256 x 256, two steps in shared memory; of 128 x 128, two steps (two workgroups a compute unit) or four (one: a step's loads
// have three steps' time to arrive).  All of 8 wavefronts: with 4 the 128 x 128 ones take 1.1 to 1.4 times as long, since nothing
// runs while a wavefront issues loads.  And of 64 x 64 by 4 wavefronts, four steps, two workgroups a compute unit, where the others are too few:
// 37 tokens, 2,048 x 5,504, forward 27 us (128 x 128: 34), 64 tokens of a whole step at 512 x 1,376 38 us (42).
enum { TILE_256 = 0, TILE_128 = 1, TILE_128_DEEP = 2, TILE_64 = 3 };
// Largest row of memory (elements) that the tile kernels take: 255 rows and a step of the next lie below Feed::OUT, so that no offset of a
// tile wraps or falls on the mark of what is outside.  Longer rows of memory are packed; a packed or internal row is as long as its columns, and
// passes with more of these are refused: width beyond GEMM_LD_MAX, or features beyond half of it (a row of dg and du).
constexpr int64_t GEMM_LD_MAX = 1 << 22;
// Launches them; false when HIP fails.  dtype: CHM_BF16 or CHM_F16.
bool gemm_launch_bf16(int products, int tile, const GemmGroup &g, void *stream);
bool gemm_launch_f16(int products, int tile, const GemmGroup &g, void *stream);
#endif

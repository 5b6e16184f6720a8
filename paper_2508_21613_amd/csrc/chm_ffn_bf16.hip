// The feed-forward block's products in bfloat16.
#include "chm_gemm.h"

bool gemm_launch_bf16(int products, int tile, const GemmGroup &g, void *stream) {
  return chm_gemm::launch<chm_gemm::Bf16>(products, tile, g, stream);
}

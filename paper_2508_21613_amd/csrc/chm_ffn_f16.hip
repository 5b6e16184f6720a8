// The feed-forward block's products in half precision.
#include "chm_gemm.h"

bool gemm_launch_f16(int products, int tile, const GemmGroup &g, void *stream) {
  return chm_gemm::launch<chm_gemm::F16>(products, tile, g, stream);
}

// The feed-forward block's products in half precision.
#include "chm_gemm.h"

bool gemm_launch_f16(int product, int tile, const GemmCall &c, void *stream) {
  return chm_gemm::launch<chm_gemm::F16>(product, tile, c, stream);
}

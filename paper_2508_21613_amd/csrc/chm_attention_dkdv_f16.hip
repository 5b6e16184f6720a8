// The gradients of attention's keys and values in float16.
#include "chm_attention_kernels.h"

using namespace chm_attention_kernels;

bool attn_dkdv_f16(const AttnCall &c, const AttnLaunch &l) { return launch_shape<F16, DKDV>(c, l); }

// The gradient of attention's queries in float16.
#include "chm_attention_kernels.h"

using namespace chm_attention_kernels;

bool attn_dq_f16(const AttnCall &c, const AttnLaunch &l) { return launch_shape<F16, DQ>(c, l); }

// The gradient of attention's queries in bfloat16.
#include "chm_attention_kernels.h"

using namespace chm_attention_kernels;

bool attn_dq_bf16(const AttnCall &c, const AttnLaunch &l) { return launch_shape<Bf16, DQ>(c, l); }

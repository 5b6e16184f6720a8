// The gradients of attention's keys and values in bfloat16.
#include "chm_attention_kernels.h"

using namespace chm_attention_kernels;

bool attn_dkdv_bf16(const AttnCall &c, const AttnLaunch &l) { return launch_shape<Bf16, DKDV>(c, l); }

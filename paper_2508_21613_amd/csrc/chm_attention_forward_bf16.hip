// Attention's forward kernels in bfloat16.
#include "chm_attention_kernels.h"

using namespace chm_attention_kernels;

bool attn_forward_bf16(const AttnCall &c, const AttnLaunch &l, bool few) { return few ? launch_shape<Bf16, FEW>(c, l) : launch_shape<Bf16, FORWARD>(c, l); }

// Attention's forward kernels in float16.
#include "chm_attention_kernels.h"

using namespace chm_attention_kernels;

bool attn_forward_f16(const AttnCall &c, const AttnLaunch &l, bool few) { return few ? launch_shape<F16, FEW>(c, l) : launch_shape<F16, FORWARD>(c, l); }

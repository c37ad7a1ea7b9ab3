// Attention over pages of 8-bit keys (attn_kernels.h has the
// kernels).
#include "attn_kernels.h"

hipError_t aio_launch_attention8(const AttnMoreArgs& a, const AttnPlan& p, int hd, int dtype,
                                 hipStream_t stream) {
  return launch_any<true, false>(a, p, hd, dtype, stream);
}

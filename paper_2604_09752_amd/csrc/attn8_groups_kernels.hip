// Attention of groups of sequences that share a prefix, over pages of 8-bit keys (attn_kernels.h has the
// kernels).
#include "attn_kernels.h"

hipError_t aio_launch_attention8_groups(const AttnMoreArgs& a, const AttnPlan& p, int hd, int dtype,
                                        hipStream_t stream) {
  return launch_any<true, true>(a, p, hd, dtype, stream);
}

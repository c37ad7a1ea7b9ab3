// Attention of groups of sequences that share a prefix, over bf16 pages (attn_kernels.h has the
// kernels).
#include "attn_kernels.h"

hipError_t aio_launch_attention_groups(const AttnMoreArgs& a, const AttnPlan& p, int hd, int dtype,
                                       hipStream_t stream) {
  return launch_any<false, true>(a, p, hd, dtype, stream);
}

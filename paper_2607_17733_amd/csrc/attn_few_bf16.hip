// attn_few_bf16.hip -- attention of few query rows over the paged cache, bf16 results
// (attn_few.h).
#include "attn_few.h"

namespace mxq {

hipError_t launch_attn_few_bf16(const AttnPagedArgs &a, int splits, int groups, hipStream_t s) {
  return launch_few<false>(a, splits, groups, s);
}

}  // namespace mxq

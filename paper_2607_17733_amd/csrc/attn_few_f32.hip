// attn_few_f32.hip -- attention of few query rows over the paged cache, float32 results
// (attn_few.h).
#include "attn_few.h"

namespace mxq {

hipError_t launch_attn_few_f32(const AttnPagedArgs &a, int splits, int groups, hipStream_t s) {
  return launch_few<true>(a, splits, groups, s);
}

}  // namespace mxq

// Attention over 8-bit pages, bfloat16 queries.
#include "paged_attend.h"

namespace frog {

hipError_t launch_paged_bf16(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream) {
    return launch_paged_type<bf16_t>(a, plan, parts, stream);
}

}  // namespace frog

// Attention over 8-bit pages, fp32 queries.
#include "paged_attend.h"

namespace frog {

hipError_t launch_paged_f32(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream) {
    return launch_paged_type<float>(a, plan, parts, stream);
}

}  // namespace frog

// Attention, forward kernels of f32 rows.
#include "attend_launch_fwd.h"

namespace frog {
template void AttendLaunch<float>::forward(const frog_attend_t&, const ForwardPlan&, char*, hipStream_t);
template void AttendLaunch<float>::shared(const frog_attend_shared_t&, const SharedPlan&, char*, hipStream_t);
}

// Attention, forward kernels of bf16 rows.
#include "attend_launch_fwd.h"

namespace frog {
template void AttendLaunch<bf16_t>::forward(const frog_attend_t&, const ForwardPlan&, char*, hipStream_t);
template void AttendLaunch<bf16_t>::shared(const frog_attend_shared_t&, const SharedPlan&, char*, hipStream_t);
}

// Attention, gradient and key-weight kernels of f32 rows.
#include "attend_launch_bwd.h"

namespace frog {
template void AttendLaunch<float>::weigh(const frog_attend_t&, const float*, char*, hipStream_t);
template void AttendLaunch<float>::backward(const frog_attend_t&, char*, hipStream_t);
}

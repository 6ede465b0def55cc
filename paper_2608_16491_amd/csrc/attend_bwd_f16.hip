// Attention, gradient and key-weight kernels of f16 rows.
#include "attend_launch_bwd.h"

namespace frog {
template void AttendLaunch<f16_t>::weigh(const frog_attend_t&, const float*, char*, hipStream_t);
template void AttendLaunch<f16_t>::backward(const frog_attend_t&, char*, hipStream_t);
}

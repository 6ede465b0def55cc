// Forward launches (included by one source file per row type).
#pragma once

#include "attend_bwd.h"
#include "attend_fwd.h"
#include "attend_launch.h"

namespace frog {

template <typename T, int D>
void launch_forward(const frog_attend_t& a, const ForwardPlan& p, char* ws, hipStream_t s) {
    const ScoreParams sp = score_params(a.scale, a.cap);
    const int group = a.heads / a.kv_heads;
    const int64_t pairs = a.batch * a.kv_heads;
    Parts parts{(float*)(ws + p.o), (float2*)(ws + p.ml), pairs * p.rows, p.splits};
    frog_attend_t b = a;
    if (a.w_out && !a.lse) b.lse = (float*)(ws + p.lse);
    const dim3 grid((unsigned)(pairs * p.splits * (p.few ? 1 : p.tiles)));
    if (p.few) {
        float* scores = a.w_out ? (float*)(ws + p.scores) : nullptr;
        if (p.groups == 1) attend_few<T, D, 1><<<grid, 256, 0, s>>>(b, sp, group, parts, scores);
        else attend_few<T, D, 2><<<grid, 256, 0, s>>>(b, sp, group, parts, scores);
    } else if (a.cap > 0.f || a.slopes || !(a.scale > 0.f)) {
        attend_tile<T, D, false, 4><<<grid, 256, 0, s>>>(b, sp, group, p.tiles, parts);
    } else {
        attend_tile<T, D, true, 4><<<grid, 256, 0, s>>>(b, sp, group, p.tiles, parts);
    }
    if (p.splits > 1) attend_join<T, D><<<dim3((unsigned)((parts.total + 3) / 4)), 256, 0, s>>>(b, group, parts);
    if (a.w_out) {
        if (p.few) attend_weigh_few<<<dim3((unsigned)((a.keys + 255) / 256 * pairs)), 256, 0, s>>>(b, group, (const float*)(ws + p.scores));
        else AttendLaunch<T>::weigh(b, b.lse, ws + p.pack, s);
    }
}

template <typename T>
void AttendLaunch<T>::forward(const frog_attend_t& a, const ForwardPlan& p, char* ws, hipStream_t s) {
    if (a.d == 32) launch_forward<T, 32>(a, p, ws, s);
    else if (a.d == 64) launch_forward<T, 64>(a, p, ws, s);
    else if (a.d == 96) launch_forward<T, 96>(a, p, ws, s);
    else launch_forward<T, 128>(a, p, ws, s);
}

}  // namespace frog

// Gradient and key-weight launches (included by one source file per row type).
#pragma once

#include "attend_bwd.h"
#include "attend_launch.h"

namespace frog {

template <typename T, int D, bool GRAD>
RowPack launch_pack(const frog_attend_t& a, const float* lse, char* pack, hipStream_t s) {
    const PackPlan p = pack_plan(a);
    const RowPack r{(float*)(pack + p.rows), (int4*)(pack + p.bounds), pack + p.zeros, (int)p.tiles};
    const int64_t waves = a.batch * a.kv_heads * p.tiles;
    pack_rows<T, D, GRAD><<<dim3((unsigned)((waves + 3) / 4)), 256, 0, s>>>(a, a.heads / a.kv_heads, r, lse);
    return r;
}

template <typename T, int D>
void launch_weigh(const frog_attend_t& a, const float* lse, char* pack, hipStream_t s) {
    const RowPack r = launch_pack<T, D, false>(a, lse, pack, s);
    const ScoreParams sp = score_params(a.scale, a.cap);
    const int tiles = (int)((a.keys + kTileRows - 1) / kTileRows);
    attend_keys<T, D, false, false, 4><<<dim3((unsigned)(a.batch * a.kv_heads * tiles)), 256, 0, s>>>(a, sp, a.heads / a.kv_heads, tiles, r);
}

template <typename T, int D>
void launch_backward(const frog_attend_t& a, char* pack, hipStream_t s) {
    const RowPack r = launch_pack<T, D, true>(a, a.lse, pack, s);
    const ScoreParams sp = score_params(a.scale, a.cap);
    const int group = a.heads / a.kv_heads;
    const int64_t rows = a.queries * group, pairs = a.batch * a.kv_heads;
    const int kt = (int)((a.keys + kTileRows - 1) / kTileRows), qt = (int)((rows + kTileRows - 1) / kTileRows);
    const dim3 kg((unsigned)(pairs * kt)), qg((unsigned)(pairs * qt));
    if (a.cap > 0.f || a.slopes) {
        if (kt) attend_keys<T, D, false, true, 4><<<kg, 256, 0, s>>>(a, sp, group, kt, r);
        attend_dq<T, D, false, 4><<<qg, 256, 0, s>>>(a, sp, group, qt, r);
    } else {
        if (kt) attend_keys<T, D, true, true, 4><<<kg, 256, 0, s>>>(a, sp, group, kt, r);
        attend_dq<T, D, true, 4><<<qg, 256, 0, s>>>(a, sp, group, qt, r);
    }
}

template <typename T>
void AttendLaunch<T>::weigh(const frog_attend_t& a, const float* lse, char* pack, hipStream_t s) {
    if (a.d == 32) launch_weigh<T, 32>(a, lse, pack, s);
    else if (a.d == 64) launch_weigh<T, 64>(a, lse, pack, s);
    else if (a.d == 96) launch_weigh<T, 96>(a, lse, pack, s);
    else launch_weigh<T, 128>(a, lse, pack, s);
}

template <typename T>
void AttendLaunch<T>::backward(const frog_attend_t& a, char* pack, hipStream_t s) {
    if (a.d == 32) launch_backward<T, 32>(a, pack, s);
    else if (a.d == 64) launch_backward<T, 64>(a, pack, s);
    else if (a.d == 96) launch_backward<T, 96>(a, pack, s);
    else launch_backward<T, 128>(a, pack, s);
}

}  // namespace frog

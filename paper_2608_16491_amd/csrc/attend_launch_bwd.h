// Gradient and key-weight launches (included by one source file per row type).
#pragma once

#include "attend_bwd.h"
#include "attend_launch.h"

namespace frog {

template <typename T, int D, bool GRAD>
RowPack launch_pack(const frog_attend_t& a, const PackPlan& p, const float* lse, char* pack, hipStream_t s) {
    const RowPack r{(float*)(pack + p.rows), (int4*)(pack + p.bounds), pack + p.zeros, (int)p.tiles};
    const int64_t waves = a.batch * a.kv_heads * p.tiles;
    const ScoreParams sp = score_params(a.scale, a.cap, a.type);
    const float shift = scores_of(a.scale, a.cap, a.slopes, a.type) == kCapped ? sp.cap2 : 0.f;
    pack_rows<T, D, GRAD><<<dim3((unsigned)((waves + 3) / 4)), 256, 0, s>>>(a, sp, a.heads / a.kv_heads, r, lse, shift);
    return r;
}

template <typename T, int D, bool GRAD>
void launch_keys(const frog_attend_t& a, const ScoreParams& sp, const PackPlan& p, const RowPack& r, char* pack, hipStream_t s) {
    const int group = a.heads / a.kv_heads, tiles = (int)((a.keys + kTileRows - 1) / kTileRows);
    const KeyParts parts{(float*)(pack + p.o), p.parts};
    const int* order = p.keys_plan.order(pack);
    if (order) schedule_keys(a, p.keys_plan, sizeof(T) == 4 && D >= 96, r.bounds, r.tiles, pack, s);
    const dim3 grid((unsigned)(a.batch * a.kv_heads * tiles * p.parts));
    by_scores<T>(scores_of(a.scale, a.cap, a.slopes, a.type), [&](auto kind) {
        attend_keys<T, D, decltype(kind)::value, GRAD, 4><<<grid, 256, 0, s>>>(a, sp, group, tiles, r, parts, order);
    });
    if (p.parts == 1) return;
    const int64_t threads = a.batch * a.kv_heads * tiles * kTileRows * (GRAD ? D / 2 : 1);
    keys_join<T, D, GRAD><<<dim3((unsigned)((threads + 255) / 256)), 256, 0, s>>>(a, sp, tiles, parts);
}

template <typename T, int D>
void launch_weigh(const frog_attend_t& a, const float* lse, char* pack, hipStream_t s) {
    const PackPlan p = pack_plan(a, false);
    const RowPack r = launch_pack<T, D, false>(a, p, lse, pack, s);
    launch_keys<T, D, false>(a, score_params(a.scale, a.cap, a.type), p, r, pack, s);
}

template <typename T, int D>
void launch_backward(const frog_attend_t& a, char* pack, hipStream_t s) {
    const PackPlan p = pack_plan(a, true);
    const RowPack r = launch_pack<T, D, true>(a, p, a.lse, pack, s);
    const ScoreParams sp = score_params(a.scale, a.cap, a.type);
    const int group = a.heads / a.kv_heads;
    const int qt = (int)((a.queries * group + kTileRows - 1) / kTileRows);
    launch_keys<T, D, true>(a, sp, p, r, pack, s);
    const int* order = p.rows_plan.order(pack);
    if (order) schedule_rows(a, p.rows_plan, sizeof(T) == 4 && D >= 128, pack, s);
    const dim3 qg((unsigned)(a.batch * a.kv_heads * qt));
    by_scores<T>(scores_of(a.scale, a.cap, a.slopes, a.type), [&](auto kind) { attend_dq<T, D, decltype(kind)::value, 4><<<qg, 256, 0, s>>>(a, sp, group, qt, r, order); });
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

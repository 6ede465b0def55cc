// Forward launches (included by one source file per row type).
#pragma once

#include <algorithm>
#include <type_traits>

#include "attend_fwd.h"
#include "attend_launch.h"

namespace frog {

template <typename T, int D>
void launch_tiles(const frog_attend_t& a, const ScoreParams& sp, int group, int tiles, const Parts& parts, const int* order, hipStream_t s) {
    const dim3 grid((unsigned)(a.batch * a.kv_heads * parts.splits * tiles));
    by_scores<T>(scores_of(a.scale, a.cap, a.slopes, a.type), [&](auto kind) {
        attend_tile<T, D, decltype(kind)::value, 4><<<grid, 256, 0, s>>>(a, sp, group, tiles, parts, order);
    });
}

template <typename T, int D>
void launch_forward(const frog_attend_t& a, const ForwardPlan& p, char* ws, hipStream_t s) {
    const ScoreParams sp = score_params(a.scale, a.cap, a.type);
    const int group = a.heads / a.kv_heads;
    const int64_t pairs = a.batch * a.kv_heads;
    const Parts parts{p.splits > 1 ? (float*)(ws + p.o) : nullptr, (float2*)(ws + p.ml), pairs * p.rows, p.splits};
    frog_attend_t b = a;
    if (a.w_out && !a.lse) b.lse = (float*)(ws + p.lse);
    if (!p.few) {
        const int* order = p.plan.order(ws);
        if (order) schedule_rows(a, p.plan, sizeof(T) == 4 && D >= 96, ws, s);
        launch_tiles<T, D>(b, sp, group, p.tiles, parts, order, s);
        if (p.splits > 1) attend_join<T, D><<<dim3((unsigned)((parts.total + 3) / 4)), 256, 0, s>>>(b, group, parts);
        if (a.w_out) AttendLaunch<T>::weigh(b, b.lse, ws + p.pack, s);
        return;
    }
    const dim3 grid((unsigned)(pairs * p.splits));
    float* scores = a.w_out ? (float*)(ws + p.scores) : nullptr;
    auto few = [&](auto plain, auto keep) {
        constexpr bool P = decltype(plain)::value, S = decltype(keep)::value;
        if (p.groups == 2) attend_few<T, D, 2, 4, P, S><<<grid, 256, 0, s>>>(b, sp, group, parts, scores);
        else if (p.splits > 1 || sizeof(T) == 4) attend_few<T, D, 1, 4, P, S><<<grid, 256, 0, s>>>(b, sp, group, parts, scores);
        else if constexpr (sizeof(T) == 2) attend_few<T, D, 1, 8, P, S><<<grid, 512, 0, s>>>(b, sp, group, parts, scores);
    };
    const bool plain = !(a.cap > 0.f) && !a.slopes;
    if (plain) a.w_out ? few(std::true_type{}, std::true_type{}) : few(std::true_type{}, std::false_type{});
    else a.w_out ? few(std::false_type{}, std::true_type{}) : few(std::false_type{}, std::false_type{});
    const int64_t joins = p.splits > 1 ? (parts.total + 3) / 4 : 0;
    if (a.w_out) attend_few_end<T, D><<<dim3((unsigned)(joins + (a.keys + 255) / 256 * pairs)), 256, 0, s>>>(b, group, parts, scores, (int)joins);
    else if (joins) attend_join<T, D><<<dim3((unsigned)joins), 256, 0, s>>>(b, group, parts);
}

template <typename T>
void AttendLaunch<T>::forward(const frog_attend_t& a, const ForwardPlan& p, char* ws, hipStream_t s) {
    if (a.d == 32) launch_forward<T, 32>(a, p, ws, s);
    else if (a.d == 64) launch_forward<T, 64>(a, p, ws, s);
    else if (a.d == 96) launch_forward<T, 96>(a, p, ws, s);
    else launch_forward<T, 128>(a, p, ws, s);
}

template <typename T, int D>
void launch_shared(const frog_attend_shared_t& a, const SharedPlan& p, char* ws, hipStream_t s) {
    const ScoreParams sp = score_params(a.scale, a.cap, a.type);
    const int group = a.heads / a.kv_heads;
    const int64_t rows = a.batch * a.heads;
    const bool plain = !(a.cap > 0.f) && !a.slopes;
    if (p.whole) {
        const dim3 grid((unsigned)p.tail_blocks);
        auto whole = [&](auto plain) {
            constexpr bool P = decltype(plain)::value;
            constexpr int W = sizeof(T) == 2 ? 8 : 4;
            if (p.groups == 1) shared_whole<T, D, 1, W, P><<<grid, 64 * W, 0, s>>>(a, sp, group);
            else shared_whole<T, D, 2, 4, P><<<grid, 256, 0, s>>>(a, sp, group);
        };
        plain ? whole(std::true_type{}) : whole(std::false_type{});
        return;
    }
    const Parts prefix{(float*)(ws + p.ho), (float2*)(ws + p.hml), rows, p.head_splits}, tail{(float*)(ws + p.to), (float2*)(ws + p.tml), rows, p.tail_splits};
    int64_t head = 0;
    if (p.few) {
        head = (int64_t)a.kv_heads * p.head_splits;
    } else if (p.head_splits) {
        // the requests are the queries of one sequence
        frog_attend_t q{};
        q.q = a.q, q.k = a.k, q.v = a.v;
        for (int i = 0; i < 2; ++i) q.q_stride[i + 1] = a.q_stride[i], q.k_stride[i + 1] = a.k_stride[i], q.v_stride[i + 1] = a.v_stride[i];
        q.lr = a.lr;
        q.batch = 1, q.queries = a.batch, q.keys = a.prefix;
        q.heads = a.heads, q.kv_heads = a.kv_heads, q.d = a.d, q.type = a.type, q.scale = a.scale, q.cap = a.cap;
        if (a.slopes) {
            q.slopes = a.slopes, q.at_q = (const float*)(ws + p.at_q), q.at_k = (const float*)(ws + p.at_k);
            shared_places<<<dim3((unsigned)((std::max(a.prefix, a.batch) + 255) / 256)), 256, 0, s>>>(a, (float*)(ws + p.at_q), (float*)(ws + p.at_k));
        }
        launch_tiles<T, D>(q, sp, group, p.tiles, prefix, nullptr, s);
    }
    if (head + p.tail_blocks > 0) {
        const dim3 grid((unsigned)(head + p.tail_blocks));
        auto few = [&](auto plain) {
            constexpr bool P = decltype(plain)::value;
            if (p.groups == 1) shared_few<T, D, 1, P><<<grid, 256, 0, s>>>(a, sp, group, (int)head, prefix, tail);
            else shared_few<T, D, 2, P><<<grid, 256, 0, s>>>(a, sp, group, (int)head, prefix, tail);
        };
        plain ? few(std::true_type{}) : few(std::false_type{});
    }
    shared_join<T, D><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, s>>>(a, group, prefix, tail);
}

template <typename T>
void AttendLaunch<T>::shared(const frog_attend_shared_t& a, const SharedPlan& p, char* ws, hipStream_t s) {
    if (a.d == 32) launch_shared<T, 32>(a, p, ws, s);
    else if (a.d == 64) launch_shared<T, 64>(a, p, ws, s);
    else if (a.d == 96) launch_shared<T, 96>(a, p, ws, s);
    else launch_shared<T, 128>(a, p, ws, s);
}

}  // namespace frog

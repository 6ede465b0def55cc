// Launches of the attention kernels of one row type (attend_bf16.hip,
// attend_f16.hip, attend_f32.hip instantiate them) and the plan they share
// with the workspace query.
#pragma once

#include <type_traits>

#include "attend_tile.h"

namespace frog {

// The order in which a pass starts the tiles of a kv head (attend_tile.h: Work).
struct SchedulePlan {
    int64_t tiles;     // of a sequence; 0: none
    int parts;         // workgroups of a tile
    int64_t at, bytes;
    int* order(char* ws) const { return tiles ? (int*)(ws + at) : nullptr; }
};

// How a forward pass is cut, by sizes alone, and where its workspace lies
// (byte offsets).
struct ForwardPlan {
    bool few;          // at most 32 query rows per kv head: no LDS tiles, 16-row products
    int groups;        // few: groups of 16 rows
    int tiles;         // else: workgroups' row tiles
    int splits;        // parts of the keys
    int64_t rows;      // query rows per (sequence, kv head)
    int64_t lse, o, ml, scores, pack;   // workspace
    SchedulePlan plan;
    int64_t bytes;
};
ForwardPlan forward_plan(const frog_attend_t& a);

// The same of a pass over a shared prefix.
struct SharedPlan {
    bool whole;               // one launch without parts
    bool few;                 // at most 32 query rows per kv head over the prefix
    int groups;               // groups of 16 rows of the few-rows passes
    int tiles;                // else: workgroups' row tiles over the prefix
    int head_splits, tail_splits;
    int64_t tail_blocks;      // workgroups of the tails
    int64_t ho, hml, to, tml, at_q, at_k;
    int64_t bytes;
};
SharedPlan shared_plan(const frog_attend_shared_t& a);

// What pack_rows prepares: offsets from the start of the region
// and how the passes that own keys are cut
struct PackPlan {
    int64_t tiles, rows, bounds, zeros, o, bytes;
    int parts;                // of the query rows, the same of every key tile
    SchedulePlan keys_plan, rows_plan;
};
PackPlan pack_plan(const frog_attend_t& a, bool grad);

// Write the schedule of tiles of kTileRows query rows, or of as many keys
// (bounds, row_tiles: RowPack).  alone: a CU holds one workgroup of the pass.
void schedule_rows(const frog_attend_t& a, const SchedulePlan& p, bool alone, char* ws, hipStream_t s);
void schedule_keys(const frog_attend_t& a, const SchedulePlan& p, bool alone, const int4* bounds, int row_tiles, char* ws, hipStream_t s);

// f(a constant of this kind), for rows of type T (fp32 rows are never kCapped)
template <typename T, typename F>
void by_scores(Scores kind, F&& f) {
    if (kind == kPlain) f(std::integral_constant<Scores, kPlain>{});
    else if (kind == kCapped) {
        if constexpr (sizeof(T) == 2) f(std::integral_constant<Scores, kCapped>{});
    } else if (kind == kBiased) f(std::integral_constant<Scores, kBiased>{});
    else f(std::integral_constant<Scores, kAny>{});
}

template <typename T>
struct AttendLaunch {
    static void forward(const frog_attend_t& a, const ForwardPlan& p, char* ws, hipStream_t s);
    static void shared(const frog_attend_shared_t& a, const SharedPlan& p, char* ws, hipStream_t s);
    // w_out from the log sums of a forward pass (natural logarithm)
    static void weigh(const frog_attend_t& a, const float* lse, char* pack, hipStream_t s);
    static void backward(const frog_attend_t& a, char* pack, hipStream_t s);
};

}  // namespace frog

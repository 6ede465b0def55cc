// Attention over rows in attribute order: argument views and device helpers
// shared by the forward, backward, shared-prefix and eviction kernels.
//
// Scores are kept in log2 units, so that a weight is one exp2: with dot = q.k,
//   no cap:  z2 = log2e scale dot - slope2 |aq - ak|
//   capped:  cap tanh(x / cap) = cap (1 - 2 / (1 + exp(2 x / cap))), so
//            z2 = capL - 2 capL / (1 + exp2(c1 dot)) - ...,
//            c1 = 2 log2e scale / cap, capL = log2e cap
// (exp2 overflows to inf and underflows to 0 where the tanh is 1 and -1).
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <cstdint>

#include "frog_internal.h"

namespace frog {

constexpr float kLog2e = 1.44269504088896340736f;
// Largest distance of one key (query) row from the next, in bytes: 64 rows
// stay within 32-bit offsets.
constexpr int64_t kMaxTokenStride = (int64_t)1 << 24;
constexpr float kLn2 = 0.69314718055994530942f;

// element types of the rows
using bf16_t = __bf16;
using f16_t = _Float16;

template <typename T, int N>
using vec = T __attribute__((ext_vector_type(N)));

struct ScoreParams {
    float mul;    // no cap: log2e scale; capped: c1
    float cap2;   // capL, 0: no cap
    float scale;
};

inline ScoreParams score_params(float scale, float cap) {
    ScoreParams s;
    s.scale = scale;
    s.cap2 = cap > 0.f ? cap * kLog2e : 0.f;
    s.mul = cap > 0.f ? 2.f * kLog2e * scale / cap : kLog2e * scale;
    return s;
}

// What a kernel is built for: no cap and no bias (the scale is then part of the
// exponent's multiply-add), one of them, or whatever the arguments say.  A
// test of the arguments between two products keeps the one's arithmetic from
// running beside the other: with it the forward pass of a long biased prompt
// took 1.37 ms instead of 1.28.
enum Scores { kPlain, kCapped, kBiased, kAny };

inline Scores scores_of(bool cap, bool bias, bool positive) {
    if (cap) return bias ? kAny : kCapped;
    return bias ? kBiased : positive ? kPlain : kAny;
}

template <Scores S>
__device__ inline bool capped(const ScoreParams& s) {
    return S == kCapped || (S == kAny && s.cap2 > 0.f);
}
template <Scores S>
__device__ inline bool biased(const void* slopes) {
    return S == kBiased || (S == kAny && slopes);
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }

// z2 of a product, without the distance bias
template <bool CAP>
__device__ inline float score2(const ScoreParams& s, float dot) {
    if constexpr (!CAP) return dot * s.mul;
    return fmaf(-2.f * s.cap2, rcp_fast(1.f + exp2_fast(dot * s.mul)), s.cap2);
}

// launchers (attend.hip, evict.hip).  The
// arguments have been checked (attend_api.cpp); ws holds the bytes of the
// matching *_ws call.
int64_t attend_ws(const frog_attend_t& a);
int launch_attend(const frog_attend_t& a, void* ws, hipStream_t stream);
int64_t attend_bwd_ws(const frog_attend_t& a);
int launch_attend_bwd(const frog_attend_t& a, void* ws, hipStream_t stream);
int64_t attend_shared_ws(const frog_attend_shared_t& a);
int launch_attend_shared(const frog_attend_shared_t& a, void* ws, hipStream_t stream);
int64_t evict_ws(const frog_evict_t& a);
int launch_evict(const frog_evict_t& a, void* ws, hipStream_t stream);

}  // namespace frog

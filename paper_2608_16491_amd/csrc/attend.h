// Attention over rows in attribute order: argument views and device helpers
// shared by the forward, backward, shared-prefix and eviction kernels.
//
// Scores are kept in log2 units, so that a weight is one exp2: with dot = q.k,
//   no cap:  z2 = log2e scale dot - slope2 |aq - ak|
//   capped:  cap tanh(x / cap) = cap (1 - 2 / (1 + exp(2 x / cap))), so
//            z2 = capL - 2 capL / (1 + exp2(c1 dot)) - ...,
//            c1 = 2 log2e scale / cap, capL = log2e cap
// (exp2 overflows to inf and underflows to 0 where the tanh is 1 and -1).
// This is within about 1.5e-7 capL of the tanh: of no account for 16-bit rows
// and the usual caps (capL = 72: 1e-5), too much for fp32 rows or a cap far
// above the scores, where small arguments take the tanh's series instead
// (ScoreParams::fine).
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <algorithm>
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
    int fine;     // capped: the tanh to a few units of its own last place
};

constexpr float kCoarseCap = 64.f;   // largest cap of 16-bit rows without the series
inline bool fine_cap(float cap, int type) { return cap > 0.f && (type == FROG_STORAGE_F32 || cap > kCoarseCap); }

inline ScoreParams score_params(float scale, float cap, int type) {
    ScoreParams s;
    s.scale = scale;
    s.fine = fine_cap(cap, type);
    s.cap2 = cap > 0.f ? cap * kLog2e : 0.f;
    s.mul = cap > 0.f ? 2.f * kLog2e * scale / cap : kLog2e * scale;
    return s;
}

// What a kernel is built for: no cap and no bias (the scale is then part of the
// exponent's multiply-add), one of them, or whatever the arguments say.  A
// test of the arguments between two products keeps the one's arithmetic from
// running beside the other: with it the forward pass of a long biased prompt
// took 1.37 ms instead of 1.28.  (kPlain masks before it scales: it wants a
// scale above 0.)
enum Scores { kPlain, kCapped, kBiased, kAny };

inline Scores scores_of(float scale, float cap, bool bias, int type) {
    if (cap > 0.f) return bias || fine_cap(cap, type) ? kAny : kCapped;
    return bias ? kBiased : scale > 0.f ? kPlain : kAny;
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
// a weight from its logarithm; at most 1, whatever the rounding of a log sum of
// great magnitude left above 0 (the exponential's own output modifier)
__device__ inline float weight2(float x) { return __builtin_amdgcn_fmed3f(exp2_fast(x), 0.f, 1.f); }
__device__ inline float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }

// capL tanh(x / cap), given y = 2 log2e x / cap and r = 1 / (1 + exp2(y)): where
// |x / cap| = |w| is below 0.35 by w - w^3/3 + 2 w^5/15 - 17 w^7/315 + 62 w^9/2835 (the
// next term is below 3e-7 of it), elsewhere by 1 - 2 r.
__device__ inline float fine_tanh(const ScoreParams& s, float y, float r) {
    const float w = y * (0.5f * kLn2), w2 = w * w;
    float t = fmaf(w2, 62.f / 2835.f, -17.f / 315.f);
    t = fmaf(w2, t, 2.f / 15.f);
    t = fmaf(w2, t, -1.f / 3.f);
    t = fmaf(w2 * w, t, w);
    return s.cap2 * (fabsf(w) < 0.35f ? t : fmaf(-2.f, r, 1.f));
}

// r of N products (kCapped: z2 = capL - 2 capL r is left to the exponent's
// multiply-add, and the largest score is the one of the least r)
template <int N, typename V>
__device__ inline void cap_shares(const ScoreParams& s, V& z) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = rcp_fast(1.f + exp2_fast(z[i] * s.mul));
}

// capped z2 of N products, without the distance bias
template <int N, typename V>
__device__ inline void cap_scores(const ScoreParams& s, V& z) {
    if (s.fine) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = z[i] * s.mul;
            z[i] = fine_tanh(s, y, rcp_fast(1.f + exp2_fast(y)));
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = fmaf(-2.f * s.cap2, rcp_fast(1.f + exp2_fast(z[i] * s.mul)), s.cap2);
    }
}

// launch(first, grid) for `total` workgroups, as many at a time as a launch takes
// (fewer than 2^32 threads); nothing follows a launch that failed.
template <typename F>
inline hipError_t in_launches(int64_t total, int threads, F&& launch) {
    const int64_t most = 0xffffffffll / threads;
    for (int64_t first = 0; first < total; first += most) {
        launch(first, dim3((unsigned)std::min(most, total - first)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// launchers (attend.hip, evict.hip).  The
// arguments have been checked (attend_api.cpp), and the matching *_ws call, which
// gives the bytes of ws, has not refused the call's grids (a negative FROG_E*).
int64_t attend_ws(const frog_attend_t& a);
int launch_attend(const frog_attend_t& a, void* ws, hipStream_t stream);
int64_t attend_bwd_ws(const frog_attend_t& a);
int launch_attend_bwd(const frog_attend_t& a, void* ws, hipStream_t stream);
int64_t attend_shared_ws(const frog_attend_shared_t& a);
int launch_attend_shared(const frog_attend_shared_t& a, void* ws, hipStream_t stream);
int64_t evict_ws(const frog_evict_t& a);
int launch_evict(const frog_evict_t& a, void* ws, hipStream_t stream);

}  // namespace frog

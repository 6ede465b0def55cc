// Selection of the largest of a list by one workgroup, and their places in
// order: the keys' 32-bit codes (which order like what they stand for) are
// sorted out by radix digits, ties going to the lowest place; every wavefront
// then lists the kept places of its piece with ballots, after one prefix sum
// over the wavefronts' counts.  Used by eviction and by the choice of pages.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace frog {

// LDS of a workgroup of BLOCK threads
template <int BLOCK>
struct PickSpace {
    static_assert(BLOCK == 1024, "three digits of 11, 11 and 10 bits, two bins a thread");
    int hist[2 * BLOCK], part[BLOCK / 64], bound[2], counts[2][BLOCK / 64];
};

// inclusive prefix sum over the workgroup (part: a value per wavefront)
template <int BLOCK>
__device__ inline int block_scan(int x, int* part) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) part[w] = x;
    __syncthreads();
    int before = 0;
#pragma unroll
    for (int i = 0; i < BLOCK / 64 - 1; ++i) before += i < w ? part[i] : 0;
    return x + before;
}

// The `want` largest of the codes code(0 .. n - 1) are those above `code` and
// the first `ties` equal to it (0 < want < n; else nothing is looked at).
struct Bound {
    uint32_t code;
    int ties;
};

template <int BLOCK, typename F>
__device__ inline Bound largest(int n, int want, F&& code_at, PickSpace<BLOCK>& s) {
    constexpr int kBins = 2 * BLOCK;
    uint32_t code = 0;
    int ties = 0;
    if (want > 0 && want < n) {
        ties = want;
        constexpr int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = shifts[pass], top = shift + bits[pass];
            s.hist[threadIdx.x] = s.hist[threadIdx.x + BLOCK] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += BLOCK) {
                const uint32_t c = code_at(i);
                if (pass == 0 || (c >> (top & 31)) == (code >> (top & 31))) atomicAdd(&s.hist[(c >> shift) & ((1u << bits[pass]) - 1)], 1);
            }
            __syncthreads();
            // two bins a thread, from the largest digit down
            const int d = kBins - 1 - 2 * (int)threadIdx.x, above = s.hist[d], sum = above + s.hist[d - 1];
            const int upto = block_scan<BLOCK>(sum, s.part), before = upto - sum;
            if (before < ties && upto >= ties) {
                const bool first = before + above >= ties;
                s.bound[0] = first ? d : d - 1;
                s.bound[1] = ties - before - (first ? 0 : above);
            }
            __syncthreads();
            code |= (uint32_t)s.bound[0] << shift;
            ties = s.bound[1];
        }
    }
    return {code, ties};
}

// The kept places of 0 .. n - 1 into `out`, ascending.  kind(i): 2 kept, 1 kept
// if among the first `ties` of its kind, 0 not kept.
template <int BLOCK, typename F>
__device__ inline void list_kept(int n, int ties, F&& kind_of, int32_t* out, PickSpace<BLOCK>& s) {
    constexpr int W = BLOCK / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // piece of the wavefront: whole groups of 64 places
    const int each = ((n + 64 * W - 1) / (64 * W)) * 64, from = min(n, wave * each), to = min(n, from + each);
    auto kind = [&](int i) { return i >= to ? 0 : kind_of(i); };
    int sure = 0, even = 0;
    for (int i = from; i < to; i += 64) {
        const int k = kind(i + lane);
        sure += __popcll(__ballot(k == 2));
        even += __popcll(__ballot(k == 1));
    }
    if (lane == 0) {
        s.counts[0][wave] = sure;
        s.counts[1][wave] = even;
    }
    __syncthreads();
    int at = 0, seen = 0;      // places listed, and equals passed, before the piece
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (i >= wave) break;
        at += s.counts[0][i];
        seen += s.counts[1][i];
    }
    at += min(seen, ties);
    const uint64_t below = (1ull << lane) - 1;
    for (int i = from; i < to; i += 64) {
        const int k = kind(i + lane);
        const uint64_t equal = __ballot(k == 1);
        const bool in = k == 2 || (k == 1 && seen + __popcll(equal & below) < ties);
        const uint64_t kept = __ballot(in);
        if (in) out[at + __popcll(kept & below)] = i + lane;
        at += __popcll(kept);
        seen += __popcll(equal);
    }
}

}  // namespace frog

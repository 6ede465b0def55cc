// Selection of the largest of a list by one workgroup, and their places in
// order: the keys' 32-bit codes (which order like what they stand for) are
// sorted out by radix digits, ties going to the lowest place; every wavefront
// then lists the kept places of its piece with ballots, after one prefix sum
// over the wavefronts' counts.  Used by eviction and by the choice of pages.
//   Scores that fit the registers are sorted out by one histogram over their
// values instead, spread between the least and the largest: digits of the codes
// put scores of one magnitude into few bins, where LDS serves one lane at a time.
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

// inclusive prefix sum, and maximum, over a wavefront
__device__ inline int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);     // the lane before, in rows of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // a row's last lane into the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);     // lane 31 into the upper rows
    return x;
}
__device__ inline uint32_t wave_most(uint32_t u) {
    int x = (int)u;
    auto larger = [](int p, int q) { return (int)max((uint32_t)p, (uint32_t)q); };
    x = larger(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));
    x = larger(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
    return (uint32_t)__builtin_amdgcn_readlane(x, 63);
}

// Codes of scores: they order like them, -0 equals 0, NaN is the largest; 0 stands
// below every score.
constexpr uint32_t kNaNCode = 0xFFFFFFFFu, kMostCode = 0xFF7FFFFFu, kLeastCode = 0x00800000u;   // (finite: least to most)
__device__ inline uint32_t score_code(float s) {
    if (s != s) return kNaNCode;
    const uint32_t u = __float_as_uint(s + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float score_of(uint32_t code) { return __uint_as_float(code & 0x80000000u ? code ^ 0x80000000u : ~code); }

// LDS of pick_few
template <int BLOCK>
struct FewSpace {
    static_assert(BLOCK == 1024, "two bins a thread");
    static constexpr int kBins = 2 * BLOCK, kRanked = 128;
    int hist[kBins], sums[BLOCK / 64], ends[2][BLOCK / 64], kept[2][BLOCK / 64], counts[3][8];
    int bin, inside, tied, listed;
    uint32_t codes[kRanked];
    int places[kRanked];
};

// The places of the `want` largest of 0 .. n - 1, counted from `first`, into `out`,
// ascending (0 < want <= n): n is at most BLOCK R; code[r] of lane l of wavefront w
// stands for place 64 (w R + r) + l, and places at or past n hold the code 0.
// Equal codes: the lower place.
template <int BLOCK, int R>
__device__ inline void pick_few(const uint32_t (&code)[R], int n, int want, int first, int32_t* out, FewSpace<BLOCK>& s) {
    constexpr int W = BLOCK / 64;
    using S = FewSpace<BLOCK>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, base = 64 * R * wave + lane;
    bool in[R];
#pragma unroll
    for (int r = 0; r < R; ++r) in[r] = base + 64 * r < n;
    if (want < n) {
        // ends of the finite scores (the least as a largest complement)
        uint32_t least = 0, most = 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (code[r] >= kLeastCode && code[r] <= kMostCode) least = max(least, ~code[r]), most = max(most, code[r]);
        least = wave_most(least);
        most = wave_most(most);
        if (lane == 0) s.ends[0][wave] = (int)least, s.ends[1][wave] = (int)most;
        s.hist[threadIdx.x] = s.hist[threadIdx.x + BLOCK] = 0;
        if (threadIdx.x < 24) (&s.counts[0][0])[threadIdx.x] = 0;
        if (threadIdx.x == 0) s.listed = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i) least = max(least, (uint32_t)s.ends[0][i]), most = max(most, (uint32_t)s.ends[1][i]);
        // (each step of a score's way to its bin keeps the order of two scores)
        const float low = most ? score_of(~least) : 0.f, step = most ? (score_of(most) - low) / (S::kBins - 1) : 0.f;
        const float per = step > 0.f && step < 1e38f ? fminf(1.f / step, 1e38f) : 0.f;
        int bin[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float at = (score_of(code[r]) - low) * per;
            bin[r] = code[r] > kMostCode ? S::kBins - 1 : code[r] < kLeastCode ? 0 : min(max((int)fminf(at, (float)S::kBins), 0), S::kBins - 1);
            if (in[r]) atomicAdd(&s.hist[bin[r]], 1);
        }
        __syncthreads();
        // two bins a thread, from the largest down: the one that holds the want-th
        const int d = S::kBins - 1 - 2 * (int)threadIdx.x, above = s.hist[d], under = s.hist[d - 1];
        int upto = wave_scan(above + under);
        if (lane == 63) s.sums[wave] = upto;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i) upto += i < wave ? s.sums[i] : 0;
        const int before = upto - above - under;
        if (before < want && upto >= want) {
            const bool upper = before + above >= want;
            s.bin = upper ? d : d - 1;
            s.inside = upper ? above : under;
            s.tied = want - before - (upper ? 0 : above);
        }
        __syncthreads();
        const int cut = s.bin, inside = s.inside, tied = s.tied;
        if (inside == tied) {
#pragma unroll
            for (int r = 0; r < R; ++r) in[r] = in[r] && bin[r] >= cut;
        } else if (inside <= S::kRanked) {
            // the bin's own order: a score's rank is the number of those that go before it
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (in[r] && bin[r] == cut) {
                    const int i = atomicAdd(&s.listed, 1);
                    s.codes[i] = code[r];
                    s.places[i] = base + 64 * r;
                }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (in[r] && bin[r] == cut) {
                    int rank = 0;
                    for (int i = 0; i < inside; ++i) rank += s.codes[i] > code[r] || (s.codes[i] == code[r] && s.places[i] < base + 64 * r);
                    in[r] = rank < tied;
                } else {
                    in[r] = in[r] && bin[r] > cut;
                }
            }
        } else {
            // many scores in one bin: its last code kept, three bits at a time, by counting with ballots
            uint32_t from = 0;
            int turn = 0;
            for (int shift = 30; shift >= 0; shift -= 3) {
                int mine = 0;
#pragma unroll
                for (int j = 1; j < 8; ++j) {
                    int c = 0;
#pragma unroll
                    for (int r = 0; r < R; ++r) c += __popcll(__ballot(in[r] && bin[r] == cut && code[r] >= (uint64_t)from + ((uint64_t)j << shift)));
                    mine = lane == j ? c : mine;
                }
                if (lane < 8 && mine) atomicAdd(&s.counts[turn][lane], mine);
                __syncthreads();
                int digit = 0;
#pragma unroll
                for (int j = 1; j < 8; ++j) digit = s.counts[turn][j] >= tied ? j : digit;
                from += (uint32_t)digit << shift;
                // (all have read the counts of the round before: they are cleared for the next but one)
                if (threadIdx.x < 8) s.counts[turn == 0 ? 2 : turn - 1][threadIdx.x] = 0;
                turn = turn == 2 ? 0 : turn + 1;
            }
            int sure = 0, even = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                sure += __popcll(__ballot(in[r] && bin[r] == cut && code[r] > from));
                even += __popcll(__ballot(in[r] && bin[r] == cut && code[r] == from));
            }
            if (lane == 0) s.kept[0][wave] = sure, s.kept[1][wave] = even;
            __syncthreads();
            int left = tied, seen = 0;           // equals to be kept, and equals before the wavefront
#pragma unroll
            for (int i = 0; i < W; ++i) {
                left -= s.kept[0][i];
                seen += i < wave ? s.kept[1][i] : 0;
            }
            const uint64_t below = (1ull << lane) - 1;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool equal = in[r] && bin[r] == cut && code[r] == from;
                const uint64_t equals = __ballot(equal);
                in[r] = in[r] && (bin[r] > cut || (bin[r] == cut && (code[r] > from || (equal && seen + __popcll(equals & below) < left))));
                seen += __popcll(equals);
            }
            __syncthreads();
        }
    }
    int mine = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) mine += __popcll(__ballot(in[r]));
    if (lane == 0) s.kept[0][wave] = mine;
    __syncthreads();
    int at = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) at += i < wave ? s.kept[0][i] : 0;
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint64_t kept = __ballot(in[r]);
        if (in[r]) out[at + __popcll(kept & below)] = first + base + 64 * r;
        at += __popcll(kept);
    }
}

}  // namespace frog

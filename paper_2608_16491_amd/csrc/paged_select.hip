// The pages worth a token's look (include/frog.h: frog_select_pages).
//
// A page's score is an upper bound of the scores of its rows, summed over the
// kv head's query heads:
//   S = sum_h sum_d max(q_hd least_d, q_hd largest_d) = sum_d (Q+_d largest_d + Q-_d least_d)
// with Q+ (Q-) the sum of the heads' positive (negative) parts, so a page costs
// two multiply-adds a channel whatever the group.  They are done in 64 bits and
// rounded once: which page is the last one chosen does not depend on the order of
// a sum.  The last score kept is then found among their codes (pick.h).
// Bound by the read of the bounds, 4 d bytes a page and kv head: 48 requests of up to
// 60,000 rows in pages of 32, 8 kv heads, d = 128, 185 MB: scores 39 us (4.8 TB/s; the 64-bit
// arithmetic keeps vector instructions busy 53 % of the time), the choice 7.  One
// request of 20,001 rows in pages of 64, in one launch: 9.1.

#include "paged.h"
#include "pick.h"

namespace frog {
namespace {

constexpr int kBlock = 1024;
constexpr int kFused = 512;        // most pages of a request scored and chosen by one workgroup
constexpr int kChunk = 128 * 128;   // else: channels of a workgroup's pages (of d = 128: 64 pages 43 us, 128 39.6, 256 55, 48 requests to 1,875 pages)
constexpr int kScoreBlock = 256;
template <int CTRL>
__device__ inline double moved(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// sum over the L lanes of a row (4, 8 or 16, aligned), in all of them
template <int L>
__device__ inline double row_sum(double x) {
    x += moved<0xB1>(x);
    x += moved<0x4E>(x);
    if constexpr (L >= 8) x += moved<0x141>(x);
    if constexpr (L >= 16) x += moved<0x140>(x);
    return x;
}

// What request b's lists are made of: `n` pages hold rows; `want` are listed; of
// those from `from` on `count` have to be scored, of which `pick` are taken.
struct Lists {
    int n, want, from, count, pick;
    __device__ inline Lists(const frog_select_pages_t& a, int64_t b) {
        n = (int)((rows_of(a.lengths, b, a.pages_per_request, a.cache.page) + a.cache.page - 1) >> shift_of(a.cache.page));
        want = (int)min((int64_t)n, a.keep);
        const bool all = n <= a.keep;
        from = all ? 0 : (int)a.first;
        count = all ? 0 : n - from - (int)a.recent;
        pick = all ? 0 : want - from - (int)a.recent;
        if (pick == 0) count = 0;
    }
};

// Q+ and Q- of (request b, kv head h) into LDS
template <typename T, int D>
__device__ inline void sum_queries(const frog_select_pages_t& a, int64_t b, int h, double (&parts)[2][D]) {
    const int i = threadIdx.x, group = a.heads / a.cache.kv_heads;
    if (i < D) {
        const T* q = (const T*)a.q + b * a.q_stride[0] + (int64_t)h * group * a.q_stride[1] + i;
        double up = 0.0, down = 0.0;
        for (int g0 = 0; g0 < group; g0 += 8) {      // eight heads' loads at a time
            float x[8];
#pragma unroll
            for (int g = 0; g < 8; ++g) x[g] = (float)q[(int64_t)min(g0 + g, group - 1) * a.q_stride[1]];
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                // (a NaN goes into both)
                const float y = g0 + g < group ? x[g] : 0.f;
                up += y < 0.f ? 0.0 : (double)y;
                down += y > 0.f ? 0.0 : (double)y;
            }
        }
        parts[0][i] = up;
        parts[1][i] = down;
    }
    __syncthreads();
}

// Codes of pages p0 .. p1 - 1 of (request b, kv head h) by WAVES wavefronts, put(p, code) from one lane each.
template <typename T, int D, int WAVES, typename F>
__device__ inline void score_pages(const frog_select_pages_t& a, int64_t b, int h, int p0, int p1, double (&parts)[2][D], F&& put) {
    using S = RowSplit<D>;
    constexpr int C = S::kEach, U = D == 96 ? 2 : 4;      // U pages of a row of lanes in flight
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane / S::kLanes, at = (lane % S::kLanes) * C;
    const int32_t* table = a.pages + b * a.pages_per_request;
    const uint16_t* bounds = (const uint16_t*)a.cache.bounds + (int64_t)h * 2 * D + at;
    const int64_t stride = (int64_t)a.cache.kv_heads * 2 * D;
    constexpr int kApart = WAVES * S::kRows;
    struct Pages {
        int page[U];
        Words<C / 2> least[U], most[U];
    };
    auto look = [&](int (&page)[U], int p) {
#pragma unroll
        for (int u = 0; u < U; ++u) page[u] = table[min(p + u * kApart + sub, p1 - 1)];
    };
    auto fetch = [&](Pages& x) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint16_t* src = bounds + max((int64_t)0, min((int64_t)x.page[u], a.cache.num_pages - 1)) * stride;
            x.least[u] = load_words<C / 2>(src);
            x.most[u] = load_words<C / 2>(src + D);
        }
    };
    // page numbers two steps ahead, bounds one: what the workgroup waits for first is on its way beside the queries
    Pages now, next;
    int p = p0 + w * S::kRows;
    look(now.page, p);
    look(next.page, p + U * kApart);
    fetch(now);
    sum_queries<T, D>(a, b, h, parts);
    double up[C], down[C];
#pragma unroll
    for (int i = 0; i < C; ++i) up[i] = parts[0][at + i], down[i] = parts[1][at + i];
    for (; p < p1; p += U * kApart) {
        int far[U];
        if (p + U * kApart < p1) {
            fetch(next);
            look(far, p + 2 * U * kApart);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p + u * kApart >= p1) break;
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < C / 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x = now.least[u].w[i], y = now.most[u].w[i];
                    s = __builtin_fma(down[2 * i + e], (double)__uint_as_float(e ? x & 0xFFFF0000u : x << 16), s);
                    s = __builtin_fma(up[2 * i + e], (double)__uint_as_float(e ? y & 0xFFFF0000u : y << 16), s);
                }
            s = row_sum<S::kLanes>(s);
            const int i = p + u * kApart + sub;
            if (at == 0 && i < p1) put(i, now.page[u] < 0 || now.page[u] >= a.cache.num_pages ? 0u : score_code((float)s));
        }
        now = next;
#pragma unroll
        for (int u = 0; u < U; ++u) next.page[u] = far[u];
    }
}

// the pages of list x that are chosen whatever their score, and the end of the list
__device__ inline void put_sure(const frog_select_pages_t& a, int64_t x, const Lists& l) {
    int32_t* out = a.chosen + x * a.keep;
    const int recent = l.want - l.from - l.pick;      // (all of them, where all are listed)
    for (int i = threadIdx.x; i < l.from; i += kBlock) out[i] = i;
    for (int i = threadIdx.x; i < recent; i += kBlock) out[l.from + l.pick + i] = l.n - recent + i;
    for (int64_t i = l.want + threadIdx.x; i < a.keep; i += kBlock) out[i] = -1;
}

// One workgroup a (request, kv head), the codes in LDS.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void select_whole(frog_select_pages_t a, int64_t first) {
    __shared__ FewSpace<kBlock> space;
    __shared__ uint32_t codes[kFused];
    __shared__ double parts[2][D];
    const int64_t x = first + blockIdx.x, b = (uint32_t)x / (uint32_t)a.cache.kv_heads;
    const Lists l(a, b);
    put_sure(a, x, l);
    if (l.count == 0) return;
    score_pages<T, D, kBlock / 64>(a, b, (int)((uint32_t)x % (uint32_t)a.cache.kv_heads), l.from, l.from + l.count, parts, [&](int p, uint32_t c) { codes[p - l.from] = c; });
    __syncthreads();
    constexpr int R = 1;
    static_assert(kFused <= R * kBlock, "a code a thread");
    uint32_t code[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = 64 * (R * (threadIdx.x >> 6) + r) + (threadIdx.x & 63);
        code[r] = i < l.count ? codes[i] : 0;
    }
    pick_few<kBlock, R>(code, l.count, l.pick, l.from, a.chosen + x * a.keep + l.from, space);
}

template <typename T, int D>
__global__ __launch_bounds__(kScoreBlock) void select_score(frog_select_pages_t a, uint32_t* codes, int chunks, uint32_t first) {
    __shared__ double parts[2][D];
    const uint32_t item = first + blockIdx.x;
    const int64_t x = item / (uint32_t)chunks, b = (uint32_t)x / (uint32_t)a.cache.kv_heads;
    const Lists l(a, b);
    const int p0 = (int)(item % (uint32_t)chunks) * (kChunk / D);
    if (p0 >= l.count) return;
    uint32_t* to = codes + x * a.pages_per_request - l.from;
    score_pages<T, D, kScoreBlock / 64>(a, b, (int)((uint32_t)x % (uint32_t)a.cache.kv_heads), l.from + p0, l.from + min(l.count, p0 + kChunk / D), parts, [&](int p, uint32_t c) { to[p] = c; });
}

// R codes a thread in registers; R = 0: from memory
template <int R>
__global__ __launch_bounds__(kBlock) void select_choose(frog_select_pages_t a, const uint32_t* codes, int64_t first) {
    __shared__ typename std::conditional<R == 0, PickSpace<kBlock>, FewSpace<kBlock>>::type space;
    const int64_t x = first + blockIdx.x;
    const Lists l(a, (uint32_t)x / (uint32_t)a.cache.kv_heads);
    put_sure(a, x, l);
    if (l.count == 0) return;
    const uint32_t* from = codes + x * a.pages_per_request;
    int32_t* out = a.chosen + x * a.keep + l.from;
    if constexpr (R == 0) {
        const Bound bound = largest<kBlock>(l.count, l.pick, [&](int i) { return from[i]; }, space);
        list_kept<kBlock>(l.count, bound.ties, [&](int i) { return from[i] > bound.code ? 2 : from[i] == bound.code ? 1 : 0; }, out, space);
        // (the list counts from the first page scored)
        __syncthreads();
        for (int i = threadIdx.x; i < l.pick; i += kBlock) out[i] += l.from;
    } else {
        uint32_t code[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = 64 * (R * (threadIdx.x >> 6) + r) + (threadIdx.x & 63);
            code[r] = i < l.count ? from[i] : 0;
        }
        pick_few<kBlock, R>(code, l.count, l.pick, l.from, out, space);
    }
}

int chunks_of(const frog_select_pages_t& a) { return (int)((a.pages_per_request + kChunk / a.cache.d - 1) / (kChunk / a.cache.d)); }

// One launch while one workgroup takes a request's pages.
bool whole(const frog_select_pages_t& a) { return a.pages_per_request <= kFused; }

template <typename T, int D>
hipError_t launch(const frog_select_pages_t& a, uint32_t* codes, hipStream_t stream) {
    const int64_t pairs = a.batch * a.cache.kv_heads;
    if (whole(a)) return in_launches(pairs, kBlock, [&](int64_t first, dim3 grid) { select_whole<T, D><<<grid, kBlock, 0, stream>>>(a, first); });
    const int chunks = chunks_of(a);
    const hipError_t e = in_launches(pairs * chunks, kScoreBlock, [&](int64_t first, dim3 grid) { select_score<T, D><<<grid, kScoreBlock, 0, stream>>>(a, codes, chunks, (uint32_t)first); });
    if (e != hipSuccess) return e;
    return in_launches(pairs, kBlock, [&](int64_t first, dim3 grid) {
        if (a.pages_per_request <= 2 * kBlock) select_choose<2><<<grid, kBlock, 0, stream>>>(a, codes, first);
        else if (a.pages_per_request <= 8 * kBlock) select_choose<8><<<grid, kBlock, 0, stream>>>(a, codes, first);
        else select_choose<0><<<grid, kBlock, 0, stream>>>(a, codes, first);
    });
}

template <typename T>
hipError_t launch_type(const frog_select_pages_t& a, uint32_t* codes, hipStream_t stream) {
    switch (a.cache.d) {
        case 32: return launch<T, 32>(a, codes, stream);
        case 64: return launch<T, 64>(a, codes, stream);
        case 96: return launch<T, 96>(a, codes, stream);
        default: return launch<T, 128>(a, codes, stream);
    }
}

__global__ __launch_bounds__(256) void select_nothing(frog_select_pages_t a, int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i < a.batch * a.cache.kv_heads * a.keep) a.chosen[i] = -1;
}

}  // namespace

int64_t select_pages_ws(const frog_select_pages_t& a) {
    if (a.batch == 0 || a.keep == 0 || a.cache.num_pages == 0 || whole(a)) return 0;
    if (a.batch * a.cache.kv_heads > 0xffffffffll / chunks_of(a)) return fail(FROG_EUNSUPPORTED, "more than 2^32 workgroups");
    return a.batch * a.cache.kv_heads * a.pages_per_request * 4;
}

int launch_select_pages(const frog_select_pages_t& a, void* ws, hipStream_t stream) {
    if (a.batch == 0 || a.keep == 0) return FROG_OK;
    hipError_t e;
    if (a.cache.num_pages == 0 || a.pages_per_request == 0) {
        const int64_t blocks = (a.batch * a.cache.kv_heads * a.keep + 255) / 256;
        e = in_launches(blocks, 256, [&](int64_t first, dim3 grid) { select_nothing<<<grid, 256, 0, stream>>>(a, first); });
    } else if (a.type == FROG_STORAGE_F32) e = launch_type<float>(a, (uint32_t*)ws, stream);
    else if (a.type == FROG_STORAGE_F16) e = launch_type<f16_t>(a, (uint32_t*)ws, stream);
    else e = launch_type<bf16_t>(a, (uint32_t*)ws, stream);
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "page selection launch: %s", hipGetErrorString(e));
}

}  // namespace frog

// The pages worth a token's look (include/frog.h: frog_select_pages).
//
// A page's score is an upper bound of the scores of its rows, summed over the
// kv head's query heads:
//   S = sum_h sum_d max(q_hd least_d, q_hd largest_d) = sum_d (Q+_d largest_d + Q-_d least_d)
// with Q+ (Q-) the sum of the heads' positive (negative) parts, so a page costs
// two multiply-adds a channel whatever the group.  They are done in 64 bits and
// rounded once: which page is the last one chosen does not depend on the order of
// a sum.  The scores' codes are then sorted out as eviction does with its weights.
// Bound by the read of the bounds, 4 d bytes a page and kv head.

#include "paged.h"
#include "pick.h"

namespace frog {
namespace {

constexpr int kBlock = 1024;
constexpr int kFused = 2048;        // most pages of a request scored and chosen by one workgroup
constexpr int kChunk = 128;         // else: pages a workgroup scores
constexpr int kScoreBlock = 256;
constexpr uint32_t kAlways = 0xFFFFFFFFu, kNaN = 0xFFFFFFFEu;

// codes order like the scores; -0 equals 0
__device__ inline uint32_t score_code(float s) {
    if (s != s) return kNaN;
    const uint32_t u = __float_as_uint(s + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

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

// Pages that hold rows of request b
__device__ inline int live_pages(const frog_select_pages_t& a, int64_t b) {
    return (int)((rows_of(a.lengths, b, a.pages_per_request, a.cache.page) + a.cache.page - 1) / a.cache.page);
}

// Codes of pages p0 .. p1 - 1 of (request b, kv head h) by WAVES wavefronts, put(p, code) from one lane each.
template <typename T, int D, int WAVES, typename F>
__device__ inline void score_pages(const frog_select_pages_t& a, int64_t b, int h, int n, int p0, int p1, F&& put) {
    using S = RowSplit<D>;
    constexpr int C = S::kEach, U = 4;      // U pages of a row of lanes in flight
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, sub = lane / S::kLanes, at = (lane % S::kLanes) * C;
    const int group = a.heads / a.cache.kv_heads;
    double up[C], down[C];
#pragma unroll
    for (int i = 0; i < C; ++i) up[i] = down[i] = 0.0;
    for (int g = 0; g < group; ++g) {
        float x[C];
        load_values((const T*)a.q + b * a.q_stride[0] + (int64_t)(h * group + g) * a.q_stride[1] + at, x);
#pragma unroll
        for (int i = 0; i < C; ++i) {
            // (a NaN goes into both)
            up[i] += x[i] < 0.f ? 0.0 : (double)x[i];
            down[i] += x[i] > 0.f ? 0.0 : (double)x[i];
        }
    }
    const int32_t* table = a.pages + b * a.pages_per_request;
    const uint16_t* bounds = (const uint16_t*)a.cache.bounds + (int64_t)h * 2 * D + at;
    const int64_t stride = (int64_t)a.cache.kv_heads * 2 * D;
    for (int p = p0 + w * S::kRows; p < p1; p += WAVES * S::kRows * U) {
        int page[U];
        Words<C / 2> least[U], most[U];
#pragma unroll
        for (int u = 0; u < U; ++u) page[u] = table[min(p + u * WAVES * S::kRows + sub, p1 - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint16_t* src = bounds + max((int64_t)0, min((int64_t)page[u], a.cache.num_pages - 1)) * stride;
            least[u] = load_words<C / 2>(src);
            most[u] = load_words<C / 2>(src + D);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < C / 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x = least[u].w[i], y = most[u].w[i];
                    s = __builtin_fma(down[2 * i + e], (double)__uint_as_float(e ? x & 0xFFFF0000u : x << 16), s);
                    s = __builtin_fma(up[2 * i + e], (double)__uint_as_float(e ? y & 0xFFFF0000u : y << 16), s);
                }
            s = row_sum<S::kLanes>(s);
            const int i = p + u * WAVES * S::kRows + sub;
            if (at == 0 && i < p1) {
                const bool none = page[u] < 0 || page[u] >= a.cache.num_pages;
                put(i, i < a.first || i >= n - a.recent ? kAlways : none ? 0u : score_code((float)s));
            }
        }
    }
}

// the list of (request, kv head) x from the codes of its n pages
template <typename F>
__device__ inline void choose(const frog_select_pages_t& a, int64_t x, int n, F&& code_at, PickSpace<kBlock>& space) {
    const int want = (int)min((int64_t)n, a.keep);
    int32_t* out = a.chosen + x * a.keep;
    const Bound bound = largest<kBlock>(n, want, code_at, space);
    list_kept<kBlock>(n, bound.ties, [&](int i) {
        if (want == n) return 2;
        const uint32_t c = code_at(i);
        return c > bound.code ? 2 : c == bound.code ? 1 : 0;
    }, out, space);
    for (int64_t i = want + threadIdx.x; i < a.keep; i += kBlock) out[i] = -1;
}

// One workgroup a (request, kv head), the codes in LDS.
template <typename T, int D>
__global__ __launch_bounds__(kBlock) void select_whole(frog_select_pages_t a, int64_t first) {
    __shared__ PickSpace<kBlock> space;
    __shared__ uint32_t codes[kFused];
    const int64_t x = first + blockIdx.x, b = x / a.cache.kv_heads;
    const int n = live_pages(a, b);
    if (n > a.keep) score_pages<T, D, kBlock / 64>(a, b, (int)(x % a.cache.kv_heads), n, 0, n, [&](int p, uint32_t c) { codes[p] = c; });
    __syncthreads();
    choose(a, x, n, [&](int i) { return codes[i]; }, space);
}

template <typename T, int D>
__global__ __launch_bounds__(kScoreBlock) void select_score(frog_select_pages_t a, uint32_t* codes, int chunks, int64_t first) {
    const int64_t item = first + blockIdx.x, x = item / chunks, b = x / a.cache.kv_heads;
    const int n = live_pages(a, b), p0 = (int)(item % chunks) * kChunk;
    if (p0 >= n || n <= a.keep) return;
    uint32_t* to = codes + x * a.pages_per_request;
    score_pages<T, D, kScoreBlock / 64>(a, b, (int)(x % a.cache.kv_heads), n, p0, min(n, p0 + kChunk), [&](int p, uint32_t c) { to[p] = c; });
}

__global__ __launch_bounds__(kBlock) void select_choose(frog_select_pages_t a, const uint32_t* codes, int64_t first) {
    __shared__ PickSpace<kBlock> space;
    const int64_t x = first + blockIdx.x;
    const uint32_t* from = codes + x * a.pages_per_request;
    choose(a, x, live_pages(a, x / a.cache.kv_heads), [&](int i) { return from[i]; }, space);
}

// One launch while one workgroup takes a request's pages.
bool whole(const frog_select_pages_t& a) { return a.pages_per_request <= kFused; }

template <typename T, int D>
hipError_t launch(const frog_select_pages_t& a, uint32_t* codes, hipStream_t stream) {
    const int64_t pairs = a.batch * a.cache.kv_heads;
    if (whole(a)) return in_launches(pairs, kBlock, [&](int64_t first, dim3 grid) { select_whole<T, D><<<grid, kBlock, 0, stream>>>(a, first); });
    const int chunks = (int)((a.pages_per_request + kChunk - 1) / kChunk);
    const hipError_t e = in_launches(pairs * chunks, kScoreBlock, [&](int64_t first, dim3 grid) { select_score<T, D><<<grid, kScoreBlock, 0, stream>>>(a, codes, chunks, first); });
    if (e != hipSuccess) return e;
    return in_launches(pairs, kBlock, [&](int64_t first, dim3 grid) { select_choose<<<grid, kBlock, 0, stream>>>(a, codes, first); });
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

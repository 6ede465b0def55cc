// Rows into a cache in 8-bit pages and back (include/frog.h: frog_cache_write,
// frog_cache_read).  Both move every byte once and are bound by HBM: prompts of
// 104,000 rows of 8 heads, d = 128, bf16 to e4m3 639 MB in 127 us (5.0 TB/s); 1.08 GB
// back in 209 (5.1); fp32 rows 1.06 GB in 222 (4.8).  Prompts of 8 x 8,000 rows at d = 128,
// 96, 64 and 32: 49, 46, 26.5 and 18 us, 0.91, 0.72, 0.84 and 0.62 of a copy's rate.  (d = 96
// has 8 lanes of 12 values a row, whose pieces of 24 bytes leave gaps in each load; d = 32
// 4 lanes, one of which stores a byte of power for 32 of codes; what each costs is not
// measured.)  A few rows take a chain of five loads: 5.4 us.

#include "paged.h"

namespace frog {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;

// first new row of request b
__device__ inline int64_t start_of(const frog_cache_write_t& a, int64_t b) {
    return a.starts ? max((int64_t)0, min((int64_t)a.starts[b], a.tokens)) : b * (int64_t)((uint32_t)a.tokens / (uint32_t)a.batch);      // (both below 2^31)
}

// WAVES wavefronts of a workgroup take a (page with new rows, kv head): the page's
// bounds are then their own, without atomics, and the same every run.  Request b's
// pages are work items from start / page + 2 b on, at least as many as its rows can
// meet (n rows meet at most n / page + 2 pages), so the host needs no lengths; the
// request of an item is found by a search over 64 requests at a time.  A row takes
// 4, 8 or 16 lanes, which find its largest magnitude among themselves.
template <typename T, bool INT8, int D, int WAVES>
__global__ __launch_bounds__(kBlock) void cache_write(frog_cache_write_t a, int64_t units, uint32_t first) {
    using S = RowSplit<D>;
    constexpr int C = S::kEach;
    const frog_cache_t& c = a.cache;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = w % WAVES;
    const int shift = shift_of(c.page);
    const uint32_t unit = (first + blockIdx.x) * (kWaves / WAVES) + w / WAVES;
    if (unit >= units) return;
    const uint32_t item = unit / (uint32_t)c.kv_heads;
    const int h = (int)(unit % (uint32_t)c.kv_heads);
    int64_t b = 0;
    for (int64_t len = a.batch; len > 1;) {
        const int64_t step = (len + 63) / 64, i = lane * step;
        const bool before = i < len && (start_of(a, b + i) >> shift) + 2 * (b + i) <= item;
        const int64_t at = max(0, __popcll(__ballot(before)) - 1) * step;
        b += at;
        len = min(step, len - at);
    }
    const int64_t start = start_of(a, b), count = max((int64_t)0, start_of(a, b + 1) - start);
    const int64_t length = a.lengths[b], before = length - count;       // rows the request had
    const int64_t from = max((int64_t)0, before), to = min(length, a.pages_per_request * c.page);
    const int64_t logical = (from >> shift) + ((int64_t)item - ((start >> shift) + 2 * b));
    const int64_t r0 = max(from, logical << shift), r1 = min(to, (logical + 1) << shift);
    if (logical < 0 || r0 >= r1) return;
    const int page = page_of(a.pages, b, a.pages_per_request, logical, c.num_pages);
    if (page < 0) return;

    const int64_t block = (int64_t)page * c.kv_heads + h;
    const int sub = lane / S::kLanes, at = (lane % S::kLanes) * C;
    // the page's bounds so far, on their way beside the rows: of a lane's channels,
    // or where wavefronts join, of a thread's
    const bool begun = (r0 & (c.page - 1)) == 0;
    uint16_t* const bounds = (uint16_t*)c.bounds + block * 2 * D;
    Words<C / 2> was[2];
    uint16_t was_one = 0;
    if (c.bounds && !begun) {
        if constexpr (WAVES == 1) {
#pragma unroll
            for (int t = 0; t < 2; ++t) was[t] = load_words<C / 2>(bounds + t * D + at);
        } else {
            was_one = bounds[min((int)threadIdx.x, 2 * D - 1)];
        }
    }
    float lo[C], hi[C];
#pragma unroll
    for (int i = 0; i < C; ++i) lo[i] = INFINITY, hi[i] = -INFINITY;
    int bad = 0;
    for (int64_t r = r0 + mine * S::kRows + sub; r - sub < r1; r += WAVES * S::kRows) {
        const bool live = r < r1;
        const int64_t token = start + (live ? r : r0) - before;
        const T* src[2] = {(const T*)a.k + token * a.k_stride[0] + h * a.k_stride[1] + at, (const T*)a.v + token * a.v_stride[0] + h * a.v_stride[1] + at};
        float x[2][C];
#pragma unroll
        for (int t = 0; t < 2; ++t) load_values(src[t], x[t]);
        const int64_t row = (block << shift) + (r & (c.page - 1));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < C; ++i) top = max(top, __float_as_uint(x[t][i]) & 0x7FFFFFFFu);
            top = over_row<S::kLanes>(top, [](uint32_t p, uint32_t q) { return max(p, q); });
            const int byte = power_byte<INT8>(top);
            const float down = power_of(254 - byte);
            Words<C / 4> codes;
#pragma unroll
            for (int i = 0; i < C / 4; ++i)
                codes.w[i] = byte == kNoRow ? 0 : codes_of<INT8>(x[t][4 * i] * down, x[t][4 * i + 1] * down, x[t][4 * i + 2] * down, x[t][4 * i + 3] * down);
            if (live) {
                store_streamed((uint8_t*)(t ? c.v : c.k) + row * D + at, codes);
                if (at == 0) (t ? c.v_exp : c.k_exp)[row] = (uint8_t)byte;
            }
            if (t == 0 && c.bounds && live) {
                bad |= byte == kNoRow;
                const float up = power_of(byte);
#pragma unroll
                for (int i = 0; i < C / 4; ++i) {
                    const vec<float, 4> y = values_of<INT8>(codes.w[i]) * up;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        lo[4 * i + e] = fminf(lo[4 * i + e], y[e]);
                        hi[4 * i + e] = fmaxf(hi[4 * i + e], y[e]);
                    }
                }
            }
        }
    }
    if (!c.bounds) return;
    // over the wavefront's rows (lanes of the same channels), then the wavefronts
    bool broken = __any(bad);
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int o = S::kLanes; o < 64; o <<= 1) {
            lo[i] = fminf(lo[i], __shfl_xor(lo[i], o));
            hi[i] = fmaxf(hi[i], __shfl_xor(hi[i], o));
        }
    // (a page begun at its row 0 forgets what it held)
    auto widened = [&](float x, uint32_t old, bool high) {
        const float y = begun ? x : __uint_as_float(old << 16);
        return (bf16_t)(broken || y != y ? NAN : high ? fmaxf(x, y) : fminf(x, y));
    };
    if constexpr (WAVES > 1) {
        __shared__ float ends[2][WAVES][D];
        __shared__ int any[WAVES];
        if (sub == 0) {
#pragma unroll
            for (int i = 0; i < C; ++i) ends[0][mine][at + i] = lo[i], ends[1][mine][at + i] = hi[i];
            if (lane == 0) any[mine] = broken;
        }
        __syncthreads();
        if (threadIdx.x >= 2 * D) return;
        const bool high = threadIdx.x >= D;
        const int i = threadIdx.x - (high ? D : 0);
        float x = ends[high][0][i];
#pragma unroll
        for (int n = 1; n < WAVES; ++n) x = high ? fmaxf(x, ends[1][n][i]) : fminf(x, ends[0][n][i]);
#pragma unroll
        for (int n = 0; n < WAVES; ++n) broken |= any[n] != 0;
        ((bf16_t*)bounds)[threadIdx.x] = widened(x, was_one, high);
    } else if (sub == 0) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            Words<C / 2> now;
#pragma unroll
            for (int i = 0; i < C / 2; ++i) {
                const float* x = t ? hi : lo;
                now.w[i] = __builtin_bit_cast(uint32_t, vec<bf16_t, 2>{widened(x[2 * i], was[t].w[i] & 0xFFFF, t), widened(x[2 * i + 1], was[t].w[i] >> 16, t)});
            }
            store_words(bounds + t * D + at, now);
        }
    }
}

// One workgroup 16 rows of a request (of one page) with all their heads, in the
// order of the outputs, 16 bytes of them a lane.
template <typename T, bool INT8, int D>
__global__ __launch_bounds__(kBlock) void cache_read(frog_cache_read_t a, uint32_t first) {
    constexpr int C = 16 / sizeof(T), kPieces = D / C;
    const frog_cache_t& c = a.cache;
    const int shift = shift_of(c.page);
    const uint32_t blocks = (uint32_t)((a.slots + 15) / 16), item = first + blockIdx.x;
    const int64_t b = item / blocks, s0 = (int64_t)(item % blocks) * 16;
    const int rows = (int)min((int64_t)16, a.slots - s0);
    const int64_t length = rows_of(a.lengths, b, a.pages_per_request, c.page);
    const int page = s0 < length ? page_of(a.pages, b, a.pages_per_request, s0 >> shift, c.num_pages) : -1;
    const int live = page < 0 ? 0 : (int)min((int64_t)rows, length - s0);
    const int64_t row0 = (((int64_t)max(page, 0) * c.kv_heads) << shift) + (s0 & (c.page - 1));
    T* const out[2] = {(T*)a.k + b * a.k_stride[0] + s0 * a.k_stride[1], (T*)a.v + b * a.v_stride[0] + s0 * a.v_stride[1]};
    for (uint32_t i = threadIdx.x; i < (uint32_t)(rows * c.kv_heads) * kPieces; i += kBlock) {
        const uint32_t n = i / kPieces, at = (i - n * kPieces) * C;
        const uint32_t s = n / (uint32_t)c.kv_heads, h = n - s * (uint32_t)c.kv_heads;
        const int64_t row = row0 + ((int64_t)h << shift) + s;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            vec<T, C> y = {};
            if ((int)s < live) {
                const Words<C / 4> codes = load_words<C / 4>((const uint8_t*)(t ? c.v : c.k) + row * D + at);
                const float up = power_of((t ? c.v_exp : c.k_exp)[row]);
#pragma unroll
                for (int w = 0; w < C / 4; ++w) {
                    const vec<float, 4> x = values_of<INT8>(codes.w[w]) * up;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[4 * w + e] = (T)x[e];
                }
            }
            const int64_t* stride = t ? a.v_stride : a.k_stride;
            __builtin_nontemporal_store(y, (vec<T, C>*)(out[t] + s * stride[1] + h * stride[2] + at));
        }
    }
}

// f(row type, whether codes are int8, d) as compile-time values
template <typename F>
void of_kind(int type, int storage, int d, F&& f) {
    auto width = [&](auto t, auto i8) {
        if (d == 32) f(t, i8, std::integral_constant<int, 32>());
        else if (d == 64) f(t, i8, std::integral_constant<int, 64>());
        else if (d == 96) f(t, i8, std::integral_constant<int, 96>());
        else f(t, i8, std::integral_constant<int, 128>());
    };
    auto codes = [&](auto t) {
        if (storage == FROG_CACHE_INT8) width(t, std::true_type());
        else width(t, std::false_type());
    };
    if (type == FROG_STORAGE_F32) codes(float());
    else if (type == FROG_STORAGE_F16) codes(f16_t());
    else codes(bf16_t());
}

}  // namespace

int launch_cache_write(const frog_cache_write_t& a, hipStream_t stream) {
    if (a.batch == 0 || a.tokens == 0 || a.cache.num_pages == 0 || a.pages_per_request == 0) return FROG_OK;
    const int64_t items = a.tokens / a.cache.page + 2 * a.batch;
    if (items > 0xfffffffbll / a.cache.kv_heads) return fail(FROG_EUNSUPPORTED, "more than 2^32 pages of a head");
    const int64_t units = items * a.cache.kv_heads;
    hipError_t e = hipSuccess;
    of_kind(a.type, a.cache.storage, a.cache.d, [&](auto t, auto i8, auto d) {
        auto run = [&](auto kernel, int waves) {
            const int each = kWaves / waves;
            e = in_launches((units + each - 1) / each, kBlock, [&](int64_t first, dim3 grid) { kernel<<<grid, kBlock, 0, stream>>>(a, units, (uint32_t)first); });
        };
        // a page whose rows a wavefront has in four rounds is one's alone (8 prompts to
        // 8,000 rows, 8 heads, pages of 16, d = 64: 29 us, by four 55; d = 128, pages of 32, twice
        // the rounds: 53 us, by four 47), unless there are few of them, whose time is
        // one page's (1,400 fp32 rows, 3 heads, pages of 16, d = 96: 9.9 us, by four 6.9)
        if (units >= 4096 && a.cache.page <= 4 * RowSplit<d.value>::kRows) run(cache_write<decltype(t), i8.value, d.value, 1>, 1);
        else run(cache_write<decltype(t), i8.value, d.value, kWaves>, kWaves);
    });
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "cache write launch: %s", hipGetErrorString(e));
}

int launch_cache_read(const frog_cache_read_t& a, hipStream_t stream) {
    if (a.batch == 0 || a.slots == 0) return FROG_OK;
    if (a.batch > 0xffffffffll / ((a.slots + 15) / 16)) return fail(FROG_EUNSUPPORTED, "more than 2^32 workgroups");
    hipError_t e = hipSuccess;
    of_kind(a.type, a.cache.storage, a.cache.d, [&](auto t, auto i8, auto d) {
        e = in_launches(a.batch * ((a.slots + 15) / 16), kBlock, [&](int64_t first, dim3 grid) {
            cache_read<decltype(t), i8.value, d.value><<<grid, kBlock, 0, stream>>>(a, (uint32_t)first);
        });
    });
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "cache read launch: %s", hipGetErrorString(e));
}

}  // namespace frog

// Attention over 8-bit pages: how a call is cut into workgroups, and the join of
// the parts (kernels: paged_attend.h).

#include "paged_attend.h"

namespace frog {
namespace {

constexpr int kJoin1 = 8, kJoin4 = 32;     // most parts that one wavefront, or four, join

// A query row's maximum and sum over its parts, then their outputs, D / 64 channels
// a lane, eight parts in flight: by one wavefront, or where there are many parts
// by the 16 of a workgroup, whose shares meet in LDS.
template <int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void paged_join(frog_attend_paged_t a, PagedPlan plan, PagedParts parts, int64_t first) {
    __shared__ float shares[WAVES][128];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = a.cache.d;
    const int64_t row = WAVES == 1 ? (first + blockIdx.x) * 4 + w : first + blockIdx.x;
    if (row >= parts.rows) return;
    const int64_t b = (uint32_t)row / (uint32_t)a.heads;      // (rows are fewer than 2^31)
    const int head = (int)((uint32_t)row % (uint32_t)a.heads);
    const Walk walk(a, b);
    const int live = ((int)(walk.end - walk.first) + plan.chunk - 1) / plan.chunk;
    const int each = (live + WAVES - 1) / WAVES, from = WAVES == 1 ? 0 : w * each, to = WAVES == 1 ? live : min(live, from + each);
    // (parts past the wavefront's last one repeat it, with a share of 0)
    float y[8][2], top[8];
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t at = (int64_t)min(s + i, to - 1) * parts.rows + row;
            top[i] = parts.ml[at].x;
            y[i][0] = parts.o[at * d + min(lane, d - 1)];
            y[i][1] = d > 64 ? parts.o[at * d + min(lane + 64, d - 1)] : 0.f;
        }
    };
    if (from < to) fetch(from);
    float all = kNoneSeen, total = 0.f;
    float2 ml = make_float2(kNoneSeen, 0.f);
    if (lane < live) ml = parts.ml[lane * parts.rows + row];
    all = ml.x;
    for (int s = lane + 64; s < live; s += 64) all = fmaxf(all, parts.ml[s * parts.rows + row].x);
    for (int o = 32; o; o >>= 1) all = fmaxf(all, __shfl_xor(all, o));
    total = ml.y * exp2_fast(ml.x - all);
    for (int s = lane + 64; s < live; s += 64) {
        const float2 more = parts.ml[s * parts.rows + row];
        total += more.y * exp2_fast(more.x - all);
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    float x[2] = {0.f, 0.f};
    for (int s = from; s < to;) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float share = s + i < to ? exp2_fast(top[i] - all) : 0.f;
            x[0] += share * y[i][0];
            x[1] += share * y[i][1];
        }
        s += 8;
        if (s < to) fetch(s);
    }
    if constexpr (WAVES > 1) {
        shares[w][lane] = x[0];
        shares[w][lane + 64] = x[1];
        __syncthreads();
        if (w) return;
        x[0] = x[1] = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            x[0] += shares[i][lane];
            x[1] += shares[i][lane + 64];
        }
    }
    const float scale = total == 0.f ? 0.f : 1.f / total;
    const int64_t at = b * a.out_stride[0] + head * a.out_stride[1] + lane;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (lane + 64 * i >= d) break;
        const float y = x[i] * scale;
        if (a.type == FROG_STORAGE_F32) ((float*)a.out)[at + 64 * i] = y;
        else if (a.type == FROG_STORAGE_F16) ((f16_t*)a.out)[at + 64 * i] = (f16_t)y;
        else ((bf16_t*)a.out)[at + 64 * i] = (bf16_t)y;
    }
    if (lane == 0 && a.lse) a.lse[row] = total == 0.f ? -INFINITY : (all + log2f(total)) * kLn2;
}

PagedPlan plan_of(const frog_attend_paged_t& a) {
    PagedPlan p;
    const int group = a.heads / a.cache.kv_heads;
    p.wide = a.type != FROG_STORAGE_F32 && group > 16;
    p.blocks = (group + (p.wide ? 31 : 15)) / (p.wide ? 32 : 16);
    p.tiles = (a.chosen ? a.num_chosen : a.pages_per_request) * (a.cache.page / kTile);
    if (a.cache.num_pages == 0) p.tiles = 0;
    const int64_t pairs = a.batch * a.cache.kv_heads * p.blocks;
    p.waves = 4;
    p.parts = 1;
    // one launch for up to 1,024 rows (the host's time for two is above what the
    // device saves: 1,001 rows of 4 kv heads 10.4 us, in parts 5.7 + 3.8); with two
    // column tiles, whose steps are longer and whose workgroups have four wavefronts
    // for eight, for up to 256, the least part (64 / 1 heads, d = 128, on the device: 1,000
    // rows in parts 12.2 us, whole 16.5; 500 rows 12.1 and 11.5; 250 rows 9.1)
    if (p.tiles <= (p.wide ? 0 : 64)) {
        p.waves = p.wide ? 4 : 8;
        p.chunk = 64;
        return p;
    }
    // Lists of pages are equally long: a workgroup a list, where that fills the CUs
    // (48 requests of 64 pages of 64 rows, 8 kv heads: 77 us, in two parts 76 + 5, in
    // six 82 + 5).  So are requests to 4,096 rows of many pairs, long and short ones side
    // by side (8 kv heads, 64 requests to 2,000 rows 30.4 us, in two parts 36.8; 128 to 3,000
    // 91, in three to six 89 to 108; 200 to 2,500 106, 101 to 135; 64 to 4,000 67, 64 to 85).
    if (pairs >= (a.chosen ? 256 : 512) && p.tiles <= kMostTiles) {
        p.chunk = kMostTiles;
        return p;
    }
    // Else a workgroup begins (about 4 us) for 16 to 64 tiles (1 us for 8), more of
    // them where there is more to do, since the longest request decides and the
    // parts are read again; of very large calls for 128.  A call is cut by the width of
    // its table (its lists), since the lengths are on the device: parts past a
    // request's rows end at once, but they count in this rule, and in the workspace
    // (48 to 4,000 rows, 16 / 2 heads: 19.3 us, in a table of 32,000 rows 32).
    // Tiles a part, us of a call (bf16, e4m3, requests of all lengths up to the one
    // named; fp16 and fp32 are cut alike, and at these sizes within 14 % of their
    // own best, bf16 within 12 %):
    //   rows, requests, heads, d       16     24     32     48     64     96    128
    //   60,000   1  32 / 8   128     36.4   32.8   31.0   31.5   28.5   30.0   30.0
    //   10,000   1  32 / 8   128     14.8   15.3   15.3   16.6   18.2   21.7   25.3
    //    4,000   4  32 / 8   128     14.0   14.7   14.3   16.0   17.7   21.2   24.7
    //    8,000  16  48 / 2   128     26.9   20.9   22.1   25.4   25.1   28.9   33.2
    //   16,000   8  32 / 8   128     35.0   34.5   36.0   36.0   40.2   42.4   38.7
    //    4,000  48  16 / 2   128     23.7   21.7   22.3   21.0   23.4   26.1   26.7
    //    8,000  32  32 / 8   128     70.5   65.0   64.4   63.4   66.2   67.3   75.1
    //   40,000  32  32 / 8   128    306.3  289.9  279.7  268.6  263.0  252.6  254.8
    const int64_t work = pairs * p.tiles, most = pairs <= 16 ? 64 : 48;
    const int64_t each = work > 400000 ? 128 : std::min<int64_t>(most, std::max<int64_t>(16, work / 500));
    p.parts = (int)((p.tiles + each - 1) / each);
    p.chunk = (int)((p.tiles + p.parts - 1) / p.parts + 7) / 8 * 8;
    p.parts = (int)((p.tiles + p.chunk - 1) / p.chunk);
    return p;
}

}  // namespace

int64_t attend_paged_ws(const frog_attend_paged_t& a) {
    if (a.batch == 0) return 0;
    const PagedPlan p = plan_of(a);
    if (a.batch * p.blocks * a.cache.kv_heads > 0x7fffffff / p.parts) return fail(FROG_EUNSUPPORTED, "more than 2^31 workgroups");
    return p.parts == 1 ? 0 : p.parts * a.batch * a.heads * (int64_t)(a.cache.d + 2) * 4;
}

int launch_attend_paged(const frog_attend_paged_t& args, void* ws, hipStream_t stream) {
    if (args.batch == 0) return FROG_OK;
    frog_attend_paged_t a = args;
    const PagedPlan p = plan_of(a);
    if (p.tiles == 0) a.pages_per_request = 0;      // no rows: outputs of 0
    PagedParts parts{};
    parts.rows = a.batch * a.heads;
    if (p.parts > 1) {
        parts.ml = (float2*)ws;
        parts.o = (float*)(parts.ml + p.parts * parts.rows);
    }
    hipError_t e = a.type == FROG_STORAGE_F32 ? launch_paged_f32(a, p, parts, stream) : a.type == FROG_STORAGE_F16 ? launch_paged_f16(a, p, parts, stream) : launch_paged_bf16(a, p, parts, stream);
    if (e == hipSuccess && p.parts > 1) {
        // eight parts of a row are in flight at once in a wavefront
        if (p.parts <= kJoin1)
            e = in_launches((parts.rows + 3) / 4, 256, [&](int64_t first, dim3 grid) { paged_join<1><<<grid, 256, 0, stream>>>(a, p, parts, first); });
        else if (p.parts <= kJoin4)
            e = in_launches(parts.rows, 256, [&](int64_t first, dim3 grid) { paged_join<4><<<grid, 256, 0, stream>>>(a, p, parts, first); });
        else
            e = in_launches(parts.rows, 1024, [&](int64_t first, dim3 grid) { paged_join<16><<<grid, 1024, 0, stream>>>(a, p, parts, first); });
    }
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "attention over pages launch: %s", hipGetErrorString(e));
}

}  // namespace frog

// Attention over 8-bit pages: how a call is cut into workgroups, and the join of
// the parts (kernels: paged_attend.h).

#include "paged_attend.h"

namespace frog {
namespace {

// A workgroup a row of queries: maximum and sums of its parts, then their
// outputs, D / 64 channels a lane.
__global__ __launch_bounds__(256) void paged_join(frog_attend_paged_t a, PagedPlan plan, PagedParts parts, int64_t first) {
    const int lane = threadIdx.x & 63, d = a.cache.d;
    const int64_t row = (first + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (row >= parts.rows) return;
    const int64_t b = (uint32_t)row / (uint32_t)a.heads;      // (rows are fewer than 2^31)
    const int head = (int)((uint32_t)row % (uint32_t)a.heads);
    const Walk walk(a, b);
    const int live = ((int)(walk.end - walk.first) + plan.chunk - 1) / plan.chunk;
    float all = kNoneSeen;
    for (int s = lane; s < live; s += 64) all = fmaxf(all, parts.ml[s * parts.rows + row].x);
    for (int o = 32; o; o >>= 1) all = fmaxf(all, __shfl_xor(all, o));
    float total = 0.f, x[2] = {0.f, 0.f};
    for (int s0 = 0; s0 < live; s0 += 64) {
        float2 ml = make_float2(kNoneSeen, 0.f);
        if (s0 + lane < live) ml = parts.ml[(s0 + lane) * parts.rows + row];
        const float share = exp2_fast(ml.x - all);
        total += ml.y * share;
        // (parts past the last one repeat it, with a share of 0)
        const int n = min(64, live - s0);
        for (int s = 0; s < n; s += 8) {
            float y[8][2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float* from = parts.o + ((s0 + min(s + i, n - 1)) * parts.rows + row) * d;
                y[i][0] = from[min(lane, d - 1)];
                y[i][1] = d > 64 ? from[min(lane + 64, d - 1)] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float f = s + i < n ? __shfl(share, s + i) : 0.f;
                x[0] += f * y[i][0];
                x[1] += f * y[i][1];
            }
        }
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
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
    // device saves: 1,001 rows of 4 kv heads 10.4 us, in parts 5.7 + 3.8)
    if (p.tiles <= (p.wide ? 0 : 64)) {
        p.waves = p.wide ? 4 : 8;
        p.chunk = 64;
        return p;
    }
    // Lists of pages are equally long: workgroups for every CU do (48 requests of 64
    // pages of 64 rows, 8 kv heads: 384 workgroups 77 us, in six parts 82 + 5).  Of
    // requests of all lengths many workgroups end early, and the longest one of
    // few decides (24 requests to 5,000 rows, 12 kv heads: parts of 512 to 1,024
    // rows 22 us, of 2,048 27, of 4,096 38).
    const int64_t want = a.chosen ? 384 : 1536;
    if (a.chosen && pairs >= 256 && p.tiles <= kMostTiles) {
        p.chunk = kMostTiles;
        return p;
    }
    const int64_t each = std::min<int64_t>(kMostTiles, std::max<int64_t>(8, (pairs * p.tiles + want - 1) / want));
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
    if (e == hipSuccess && p.parts > 1)
        e = in_launches((parts.rows + 3) / 4, 256, [&](int64_t first, dim3 grid) { paged_join<<<grid, 256, 0, stream>>>(a, p, parts, first); });
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "attention over pages launch: %s", hipGetErrorString(e));
}

}  // namespace frog

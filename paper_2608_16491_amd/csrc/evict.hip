// Shortening a cache to its heaviest and newest rows (include/frog.h:
// frog_evict).
//
// Weights become 32-bit codes that order like them; a radix selection in three
// digits finds the code of the last row kept and how many of its equals are,
// one workgroup per (sequence, head); every wavefront then lists the kept
// slots of its piece of the row with ballots, after one prefix sum over the
// wavefronts' counts.  A second kernel copies the rows.  The selection reads
// the weights five times, from L2 after the first; the copy is bound by HBM.
// 16 caches of 10,000 slots, 8 heads, d = 128, bf16, cut to 5,000: selection 20
// us, copy 120 (5.0 TB/s read and written).

#include "attend.h"
#include "pick.h"

namespace frog {
namespace {

constexpr int kBlock = 1024;

// Codes order like the weights; -0 equals 0; NaN is the lowest.
__device__ inline uint32_t code_of(float w) {
    if (w != w) return 0;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ inline int64_t live_rows(const frog_evict_t& a, int64_t b) { return max((int64_t)0, min((int64_t)a.lengths[b], a.slots)); }

__global__ __launch_bounds__(kBlock) void evict_pick(frog_evict_t a, int32_t* list, int64_t first) {
    __shared__ PickSpace<kBlock> space;
    const int64_t row = first + blockIdx.x, b = row / a.heads;
    const int n = (int)live_rows(a, b), keep = (int)a.keep;
    const int recent = (int)min((int64_t)n, a.recent), old = n - recent;
    const float* w = a.weights + row * a.slots;
    int32_t* out = list + row * a.keep;
    // of the `old` first rows the `want` heaviest: those above `code`, and the
    // first `ties` equal to it
    const int want = min(old, keep - recent);
    const Bound bound = largest<kBlock>(old, want, [&](int i) { return code_of(w[i]); }, space);
    list_kept<kBlock>(n, bound.ties, [&](int i) {   // 2: kept, 1: equal to the last kept, 0: not kept
        if (i >= old || want == old) return 2;
        if (want == 0) return 0;
        const uint32_t c = code_of(w[i]);
        return c > bound.code ? 2 : c == bound.code ? 1 : 0;
    }, out, space);
    for (int i = min(n, keep) + threadIdx.x; i < keep; i += kBlock) out[i] = -1;
    if (row % a.heads == 0 && threadIdx.x == 0) a.lengths_out[b] = min(n, keep);
}

__global__ __launch_bounds__(256) void evict_copy(frog_evict_t a, const int32_t* list, int size, int pieces, int64_t first) {
    const int64_t t = (first + blockIdx.x) * 256 + threadIdx.x, total = a.batch * a.keep * a.heads * pieces;
    if (t >= total) return;
    const int c = (int)(t % pieces);
    const int64_t slot_head = t / pieces;
    const int h = (int)(slot_head % a.heads);
    const int64_t s = slot_head / a.heads % a.keep, b = slot_head / a.heads / a.keep;
    const int64_t at = (b * a.heads + h) * a.keep + s;
    const int from = list[at];
    const int per = 16 / size;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (from >= 0) {
        k = *(const uint4*)((const char*)a.k + (b * a.k_stride[0] + from * a.k_stride[1] + h * a.k_stride[2] + c * per) * size);
        v = *(const uint4*)((const char*)a.v + (b * a.v_stride[0] + from * a.v_stride[1] + h * a.v_stride[2] + c * per) * size);
    }
    ((uint4*)a.k_out)[t] = k;
    ((uint4*)a.v_out)[t] = v;
    if (c == 0) {
        const int64_t old = (b * a.heads + h) * a.slots + from;
        a.weights_out[at] = from >= 0 ? a.weights[old] : 0.f;
        a.positions_out[at] = from >= 0 ? (a.positions ? a.positions[old] : from) : -1;
    }
}

__global__ void evict_nothing(frog_evict_t a) {
    const int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (b < a.batch) a.lengths_out[b] = 0;
}

}  // namespace

int64_t evict_ws(const frog_evict_t& a) { return a.batch * a.heads * a.keep * 4; }

int launch_evict(const frog_evict_t& a, void* ws, hipStream_t stream) {
    if (a.batch == 0) return FROG_OK;
    hipError_t e;
    if (a.keep == 0) {
        evict_nothing<<<dim3((unsigned)((a.batch + 255) / 256)), 256, 0, stream>>>(a);
        e = hipGetLastError();
    } else {
        const int size = a.type == FROG_STORAGE_F32 ? 4 : 2, pieces = a.d * size / 16;
        const int64_t copies = (a.batch * a.keep * a.heads * pieces + 255) / 256;
        int32_t* list = (int32_t*)ws;
        e = in_launches(a.batch * a.heads, kBlock, [&](int64_t first, dim3 grid) { evict_pick<<<grid, kBlock, 0, stream>>>(a, list, first); });
        if (e == hipSuccess) e = in_launches(copies, 256, [&](int64_t first, dim3 grid) { evict_copy<<<grid, 256, 0, stream>>>(a, list, size, pieces, first); });
    }
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "eviction launch: %s", hipGetErrorString(e));
}

}  // namespace frog

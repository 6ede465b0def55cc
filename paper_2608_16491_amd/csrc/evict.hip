// Shortening a cache to its heaviest and newest rows (include/frog.h:
// frog_evict).
//
// Weights become 32-bit codes that order like them; a radix selection finds
// the code of the last row kept and how many of its equals are, one workgroup
// per (sequence, head); a prefix sum over the slots lists the kept ones in
// slot order; the rows are copied by a second kernel.

#include "attend.h"

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

// inclusive prefix sum over the workgroup; *total receives the sum
__device__ inline int block_scan(int x, int* part, int* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) part[w] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < kBlock / 64; ++i) {
        before += i < w ? part[i] : 0;
        all += part[i];
    }
    *total = all;
    return x + before;
}

__global__ __launch_bounds__(kBlock) void evict_pick(frog_evict_t a, int32_t* list) {
    __shared__ int hist[256], part[kBlock / 64], bound[2];
    const int64_t row = blockIdx.x, b = row / a.heads;
    const int n = (int)live_rows(a, b), keep = (int)a.keep;
    const int recent = (int)min((int64_t)n, a.recent), old = n - recent;
    const float* w = a.weights + row * a.slots;
    int32_t* out = list + row * a.keep;
    // of the `old` first rows the `want` heaviest: those above `code`, and the
    // first `ties` equal to it
    const int want = min(old, keep - recent);
    uint32_t code = 0;
    int ties = want;
    if (want > 0 && want < old) {
        int left = want;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < old; i += kBlock) {
                const uint32_t c = code_of(w[i]);
                if (shift == 24 || (c >> (shift + 8)) == (code >> (shift + 8))) atomicAdd(&hist[(c >> shift) & 255], 1);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int v = 255, rest = left;
                while (v > 0 && hist[v] < rest) rest -= hist[v--];
                bound[0] = v;
                bound[1] = rest;
            }
            __syncthreads();
            code |= (uint32_t)bound[0] << shift;
            left = bound[1];
        }
        ties = left;
    } else if (want == old) {
        ties = old;
    }
    int kept = 0, seen = 0;   // rows listed, rows equal to the code passed
    for (int i0 = 0; i0 < n; i0 += kBlock) {
        const int i = i0 + threadIdx.x;
        bool in = false, tie = false;
        if (i < n) {
            if (i >= old || want == old) in = true;
            else if (want > 0) {
                const uint32_t c = code_of(w[i]);
                in = c > code;
                tie = c == code;
            }
        }
        int total;
        const int t = block_scan(tie, part, &total);
        if (tie && seen + t <= ties) in = true;
        seen += total;
        const int at = kept + block_scan(in, part, &total) - 1;
        if (in) out[at] = i;
        kept += total;
    }
    for (int i = kept + threadIdx.x; i < keep; i += kBlock) out[i] = -1;
    if (row % a.heads == 0 && threadIdx.x == 0) a.lengths_out[b] = min(n, keep);
}

__global__ __launch_bounds__(256) void evict_copy(frog_evict_t a, const int32_t* list, int size, int pieces) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, total = a.batch * a.keep * a.heads * pieces;
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
    if (a.keep == 0) {
        evict_nothing<<<dim3((unsigned)((a.batch + 255) / 256)), 256, 0, stream>>>(a);
    } else {
        const int size = a.type == FROG_STORAGE_F32 ? 4 : 2, pieces = a.d * size / 16;
        const int64_t total = a.batch * a.keep * a.heads * pieces;
        if ((total + 255) / 256 > 0x7fffffff) return fail(FROG_EUNSUPPORTED, "too many rows kept");
        evict_pick<<<dim3((unsigned)(a.batch * a.heads)), kBlock, 0, stream>>>(a, (int32_t*)ws);
        evict_copy<<<dim3((unsigned)((total + 255) / 256)), 256, 0, stream>>>(a, (const int32_t*)ws, size, pieces);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "eviction launch: %s", hipGetErrorString(e));
}

}  // namespace frog

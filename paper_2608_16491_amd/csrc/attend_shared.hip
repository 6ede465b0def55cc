// Attention of many requests over one shared prefix and their own paged tails
// (include/frog.h: frog_attend_shared).
//
// One wavefront per (request, head): its interval of the prefix, then its
// tail, 64 keys a step with the running maximum and sum of the softmax.

#include "attend.h"

namespace frog {
namespace {

constexpr int kBlock = 256;

__device__ inline float wave_max(float x) {
    for (int o = 32; o; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}
__device__ inline float wave_sum(float x) {
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

template <typename T, bool CAP>
__global__ __launch_bounds__(kBlock) void shared_rows(frog_attend_shared_t a, ScoreParams sp) {
    __shared__ float qs[4][128], ps[4][64];
    __shared__ const T* vr[4][64];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + w;
    if (row >= a.batch * a.heads) return;
    const int h = (int)(row % a.heads), hk = h / (a.heads / a.kv_heads);
    const int64_t b = row / a.heads;
    const T* q = (const T*)a.q + b * a.q_stride[0] + h * a.q_stride[1];
    for (int c = lane; c < a.d; c += 64) qs[w][c] = (float)q[c];
    int64_t lo = 0, hi = a.prefix - 1;
    if (a.lr) {
        lo = max(lo, (int64_t)a.lr[2 * b]);
        hi = min(hi, (int64_t)a.lr[2 * b + 1]);
    }
    const int64_t len = a.pages_per_request > 0 ? max((int64_t)0, min((int64_t)a.lengths[b], a.pages_per_request * a.page)) : 0;
    const int64_t head = hi >= lo ? hi - lo + 1 : 0, total = head + len;
    const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.f;
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    for (int64_t j0 = 0; j0 < total; j0 += 64) {
        const int64_t j = j0 + lane;
        const T* k = nullptr;
        const T* v = nullptr;
        int64_t at = 0;
        if (j < head) {
            at = lo + j;
            k = (const T*)a.k + at * a.k_stride[0] + hk * a.k_stride[1];
            v = (const T*)a.v + at * a.v_stride[0] + hk * a.v_stride[1];
        } else if (j < total) {
            const int64_t t = j - head, pg = a.pages[b * a.pages_per_request + t / a.page];
            at = a.prefix + t;
            if (pg >= 0 && pg < a.num_pages) {
                k = (const T*)a.k_pages + pg * a.k_pages_stride[0] + (t % a.page) * a.k_pages_stride[1] + hk * a.k_pages_stride[2];
                v = (const T*)a.v_pages + pg * a.v_pages_stride[0] + (t % a.page) * a.v_pages_stride[1] + hk * a.v_pages_stride[2];
            }
        }
        float z = -INFINITY;
        if (k) {
            float s = 0.f;
            for (int c = 0; c < a.d; ++c) s = fmaf(qs[w][c], (float)k[c], s);
            z = score2<CAP>(sp, s) - slope * fabsf((float)(a.prefix + len - 1 - at));
        }
        const float mn = fmaxf(m, wave_max(z));
        if (mn == -INFINITY) continue;
        const float p = exp2_fast(z - mn), scale = exp2_fast(m - mn);
        l = l * scale + wave_sum(p);
        m = mn;
        ps[w][lane] = p;
        vr[w][lane] = v;
        for (int u = 0; u < 2; ++u) {
            const int c = lane + 64 * u;
            if (c >= a.d) break;
            float o = acc[u] * scale;
            for (int t = 0; t < 64; ++t)
                if (vr[w][t]) o = fmaf(ps[w][t], (float)vr[w][t][c], o);
            acc[u] = o;
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* out = (T*)a.out + b * a.out_stride[0] + h * a.out_stride[1];
    for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < a.d) out[lane + 64 * u] = (T)(acc[u] * inv);
    if (a.lse && lane == 0) a.lse[row] = l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, bool CAP>
int run(const frog_attend_shared_t& a, hipStream_t stream) {
    const int64_t rows = a.batch * a.heads;
    if (rows) shared_rows<T, CAP><<<dim3((unsigned)((rows + 3) / 4)), kBlock, 0, stream>>>(a, score_params(a.scale, a.cap));
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "shared attention launch: %s", hipGetErrorString(e));
}

}  // namespace

int64_t attend_shared_ws(const frog_attend_shared_t&) { return 0; }

int launch_attend_shared(const frog_attend_shared_t& a, void*, hipStream_t stream) {
    if (a.type == FROG_STORAGE_F32) return a.cap > 0.f ? run<float, true>(a, stream) : run<float, false>(a, stream);
    if (a.type == FROG_STORAGE_F16) return a.cap > 0.f ? run<f16_t, true>(a, stream) : run<f16_t, false>(a, stream);
    return a.cap > 0.f ? run<bf16_t, true>(a, stream) : run<bf16_t, false>(a, stream);
}

}  // namespace frog

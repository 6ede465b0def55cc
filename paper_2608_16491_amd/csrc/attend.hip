// Range attention, forward (include/frog.h: frog_attend).
//
// One wavefront per (sequence, query, head): 64 keys a step, a lane each, the
// running maximum and sum of the softmax in registers, then the lanes turn to
// the values' columns.  The weights are summed per key in a second pass.

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

template <typename T>
__device__ inline float dot_row(const float* q, const T* k, int d) {
    float s = 0.f;
    for (int c = 0; c < d; ++c) s = fmaf(q[c], (float)k[c], s);
    return s;
}

template <typename T, bool CAP>
__global__ __launch_bounds__(kBlock) void attend_rows(frog_attend_t a, ScoreParams sp, float* lse) {
    __shared__ float qs[4][128], ps[4][64];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + w;
    if (row >= a.batch * a.heads * a.queries) return;
    const int64_t i = row % a.queries, bh = row / a.queries;
    const int h = (int)(bh % a.heads);
    const int64_t b = bh / a.heads;
    const int hk = h / (a.heads / a.kv_heads);
    const T* q = (const T*)a.q + b * a.q_stride[0] + i * a.q_stride[1] + h * a.q_stride[2];
    const T* k = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2];
    const T* v = (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2];
    for (int c = lane; c < a.d; c += 64) qs[w][c] = (float)q[c];
    int64_t lo = 0, hi = a.keys - 1;
    if (a.lr) {
        const int32_t* p = a.lr + b * a.lr_stride + 2 * i;
        lo = max(lo, (int64_t)p[0]);
        hi = min(hi, (int64_t)p[1]);
    }
    const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.f;
    const float aq = a.slopes ? a.at_q[b * a.at_q_stride + i] : 0.f;
    const float* ak = a.slopes ? a.at_k + b * a.at_k_stride[0] + hk * a.at_k_stride[1] : nullptr;
    float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
    for (int64_t j0 = lo; j0 <= hi; j0 += 64) {
        const int64_t j = j0 + lane;
        float z = -INFINITY;
        if (j <= hi) {
            z = score2<CAP>(sp, dot_row(qs[w], k + j * a.k_stride[1], a.d));
            if (ak) z -= slope * fabsf(aq - ak[j]);
        }
        const float mn = fmaxf(m, wave_max(z));
        const float p = j <= hi ? exp2_fast(z - mn) : 0.f, scale = exp2_fast(m - mn);
        l = l * scale + wave_sum(p);
        m = mn;
        ps[w][lane] = p;
        const int cnt = (int)min((int64_t)64, hi - j0 + 1);
        for (int u = 0; u < 2; ++u) {
            const int c = lane + 64 * u;
            if (c >= a.d) break;
            float o = acc[u] * scale;
            for (int t = 0; t < cnt; ++t) o = fmaf(ps[w][t], (float)v[(j0 + t) * a.v_stride[1] + c], o);
            acc[u] = o;
        }
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    T* out = (T*)a.out + b * a.out_stride[0] + i * a.out_stride[1] + h * a.out_stride[2];
    for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < a.d) out[lane + 64 * u] = (T)(acc[u] * inv);
    if (lse && lane == 0) lse[bh * a.queries + i] = l > 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
}

template <typename T, bool CAP>
__global__ __launch_bounds__(kBlock) void weigh_keys(frog_attend_t a, ScoreParams sp, const float* lse) {
    __shared__ float ks[4][128];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + w;
    if (row >= a.batch * a.kv_heads * a.keys) return;
    const int64_t j = row % a.keys, bh = row / a.keys;
    const int hk = (int)(bh % a.kv_heads), group = a.heads / a.kv_heads;
    const int64_t b = bh / a.kv_heads;
    const T* k = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2] + j * a.k_stride[1];
    for (int c = lane; c < a.d; c += 64) ks[w][c] = (float)k[c];
    const float ak = a.slopes ? a.at_k[b * a.at_k_stride[0] + hk * a.at_k_stride[1] + j] : 0.f;
    float sum = 0.f;
    for (int64_t r = lane; r < a.queries * group; r += 64) {
        const int64_t i = r / group;
        const int h = hk * group + (int)(r % group);
        if (a.lr) {
            const int32_t* p = a.lr + b * a.lr_stride + 2 * i;
            if (j < p[0] || j > p[1]) continue;
        }
        const T* q = (const T*)a.q + b * a.q_stride[0] + i * a.q_stride[1] + h * a.q_stride[2];
        float z = score2<CAP>(sp, dot_row(ks[w], q, a.d));
        if (a.slopes) z -= a.slopes[h] * kLog2e * fabsf(a.at_q[b * a.at_q_stride + i] - ak);
        sum += exp2_fast(z - lse[(b * a.heads + h) * a.queries + i] * kLog2e);
    }
    sum = wave_sum(sum);
    if (lane == 0) a.w_out[bh * a.keys + j] = (a.w_in ? a.w_in[bh * a.keys + j] : 0.f) + sum;
}

template <typename T, bool CAP>
int run(const frog_attend_t& a, void* ws, hipStream_t stream) {
    const ScoreParams sp = score_params(a.scale, a.cap);
    float* lse = a.lse ? a.lse : (float*)ws;
    const int64_t rows = a.batch * a.heads * a.queries, cols = a.batch * a.kv_heads * a.keys;
    if (rows) attend_rows<T, CAP><<<dim3((unsigned)((rows + 3) / 4)), kBlock, 0, stream>>>(a, sp, lse);
    if (a.w_out && cols) weigh_keys<T, CAP><<<dim3((unsigned)((cols + 3) / 4)), kBlock, 0, stream>>>(a, sp, lse);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "attention launch: %s", hipGetErrorString(e));
}

}  // namespace

int64_t attend_ws(const frog_attend_t& a) { return a.w_out && !a.lse ? a.batch * a.heads * a.queries * 4 : 0; }

int launch_attend(const frog_attend_t& a, void* ws, hipStream_t stream) {
    if (a.type == FROG_STORAGE_F32) return a.cap > 0.f ? run<float, true>(a, ws, stream) : run<float, false>(a, ws, stream);
    if (a.type == FROG_STORAGE_F16) return a.cap > 0.f ? run<f16_t, true>(a, ws, stream) : run<f16_t, false>(a, ws, stream);
    return a.cap > 0.f ? run<bf16_t, true>(a, ws, stream) : run<bf16_t, false>(a, ws, stream);
}

}  // namespace frog

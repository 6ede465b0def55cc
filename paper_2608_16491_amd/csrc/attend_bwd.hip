// Range attention, gradients (include/frog.h: frog_attend_backward).
//
// delta = dout.out per query; then one wavefront per (sequence, query, head)
// for dq and one per (sequence, key, kv head) for dk and dv, each summing in
// a fixed order.

#include "attend.h"

namespace frog {
namespace {

constexpr int kBlock = 256;

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

// (z2, d y / d x) of a product, without the bias
template <bool CAP>
__device__ inline float2 score_slope(const ScoreParams& s, float dot) {
    if constexpr (!CAP) return make_float2(dot * s.mul, s.scale);
    const float r = rcp_fast(1.f + exp2_fast(dot * s.mul));
    // tanh = 1 - 2 r, 1 - tanh^2 = 4 r (1 - r)
    return make_float2(s.cap2 - 2.f * s.cap2 * r, 4.f * r * (1.f - r) * s.scale);
}

template <typename T, bool CAP>
__global__ __launch_bounds__(kBlock) void grad_q(frog_attend_t a, ScoreParams sp, float* delta) {
    __shared__ float qs[4][128], gs[4][128], ps[4][64];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + w;
    if (row >= a.batch * a.heads * a.queries) return;
    const int64_t i = row % a.queries, bh = row / a.queries;
    const int h = (int)(bh % a.heads);
    const int64_t b = bh / a.heads;
    const int hk = h / (a.heads / a.kv_heads);
    const T* q = (const T*)a.q + b * a.q_stride[0] + i * a.q_stride[1] + h * a.q_stride[2];
    const T* g = (const T*)a.dout + b * a.dout_stride[0] + i * a.dout_stride[1] + h * a.dout_stride[2];
    const T* o = (const T*)a.out + b * a.out_stride[0] + i * a.out_stride[1] + h * a.out_stride[2];
    const T* k = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2];
    const T* v = (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2];
    float dl = 0.f;
    for (int c = lane; c < a.d; c += 64) {
        qs[w][c] = (float)q[c];
        gs[w][c] = (float)g[c];
        dl += (float)g[c] * (float)o[c];
    }
    dl = wave_sum(dl);
    if (lane == 0) delta[bh * a.queries + i] = dl;
    int64_t lo = 0, hi = a.keys - 1;
    if (a.lr) {
        const int32_t* p = a.lr + b * a.lr_stride + 2 * i;
        lo = max(lo, (int64_t)p[0]);
        hi = min(hi, (int64_t)p[1]);
    }
    const float slope = a.slopes ? a.slopes[h] * kLog2e : 0.f;
    const float aq = a.slopes ? a.at_q[b * a.at_q_stride + i] : 0.f;
    const float* ak = a.slopes ? a.at_k + b * a.at_k_stride[0] + hk * a.at_k_stride[1] : nullptr;
    const float lse = a.lse[bh * a.queries + i] * kLog2e;
    float acc[2] = {0.f, 0.f};
    for (int64_t j0 = lo; j0 <= hi; j0 += 64) {
        const int64_t j = j0 + lane;
        float dx = 0.f;
        if (j <= hi) {
            float2 z = score_slope<CAP>(sp, dot_row(qs[w], k + j * a.k_stride[1], a.d));
            if (ak) z.x -= slope * fabsf(aq - ak[j]);
            dx = exp2_fast(z.x - lse) * (dot_row(gs[w], v + j * a.v_stride[1], a.d) - dl) * z.y;
        }
        ps[w][lane] = dx;
        const int cnt = (int)min((int64_t)64, hi - j0 + 1);
        for (int u = 0; u < 2; ++u) {
            const int c = lane + 64 * u;
            if (c >= a.d) break;
            for (int t = 0; t < cnt; ++t) acc[u] = fmaf(ps[w][t], (float)k[(j0 + t) * a.k_stride[1] + c], acc[u]);
        }
    }
    T* dq = (T*)a.dq + b * a.dq_stride[0] + i * a.dq_stride[1] + h * a.dq_stride[2];
    for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < a.d) dq[lane + 64 * u] = (T)acc[u];
}

template <typename T, bool CAP>
__global__ __launch_bounds__(kBlock) void grad_kv(frog_attend_t a, ScoreParams sp, const float* delta) {
    __shared__ float ks[4][128], vs[4][128], ps[4][64], xs[4][64];
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + w;
    if (row >= a.batch * a.kv_heads * a.keys) return;
    const int64_t j = row % a.keys, bh = row / a.keys;
    const int hk = (int)(bh % a.kv_heads), group = a.heads / a.kv_heads;
    const int64_t b = bh / a.kv_heads;
    const T* k = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2] + j * a.k_stride[1];
    const T* v = (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2] + j * a.v_stride[1];
    for (int c = lane; c < a.d; c += 64) {
        ks[w][c] = (float)k[c];
        vs[w][c] = (float)v[c];
    }
    const float ak = a.slopes ? a.at_k[b * a.at_k_stride[0] + hk * a.at_k_stride[1] + j] : 0.f;
    float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
    const int64_t rows = a.queries * group;
    for (int64_t r0 = 0; r0 < rows; r0 += 64) {
        const int64_t r = r0 + lane, i = r / group;
        const int h = hk * group + (int)(r % group);
        bool in = r < rows;
        if (in && a.lr) {
            const int32_t* p = a.lr + b * a.lr_stride + 2 * i;
            in = j >= p[0] && j <= p[1];
        }
        uint64_t mask = __ballot(in);
        if (!mask) continue;
        float p = 0.f, dx = 0.f;
        if (in) {
            const T* q = (const T*)a.q + b * a.q_stride[0] + i * a.q_stride[1] + h * a.q_stride[2];
            const T* g = (const T*)a.dout + b * a.dout_stride[0] + i * a.dout_stride[1] + h * a.dout_stride[2];
            float2 z = score_slope<CAP>(sp, dot_row(ks[w], q, a.d));
            if (a.slopes) z.x -= a.slopes[h] * kLog2e * fabsf(a.at_q[b * a.at_q_stride + i] - ak);
            const int64_t at = (b * a.heads + h) * a.queries + i;
            p = exp2_fast(z.x - a.lse[at] * kLog2e);
            dx = p * (dot_row(vs[w], g, a.d) - delta[at]) * z.y;
        }
        ps[w][lane] = p;
        xs[w][lane] = dx;
        for (; mask; mask &= mask - 1) {
            const int t = __ffsll((unsigned long long)mask) - 1;
            const int64_t it = (r0 + t) / group;
            const int ht = hk * group + (int)((r0 + t) % group);
            const T* q = (const T*)a.q + b * a.q_stride[0] + it * a.q_stride[1] + ht * a.q_stride[2];
            const T* g = (const T*)a.dout + b * a.dout_stride[0] + it * a.dout_stride[1] + ht * a.dout_stride[2];
            for (int u = 0; u < 2; ++u) {
                const int c = lane + 64 * u;
                if (c >= a.d) break;
                dk[u] = fmaf(xs[w][t], (float)q[c], dk[u]);
                dv[u] = fmaf(ps[w][t], (float)g[c], dv[u]);
            }
        }
    }
    T* pk = (T*)a.dk + b * a.dk_stride[0] + hk * a.dk_stride[2] + j * a.dk_stride[1];
    T* pv = (T*)a.dv + b * a.dv_stride[0] + hk * a.dv_stride[2] + j * a.dv_stride[1];
    for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < a.d) {
            pk[lane + 64 * u] = (T)dk[u];
            pv[lane + 64 * u] = (T)dv[u];
        }
}

template <typename T, bool CAP>
int run(const frog_attend_t& a, void* ws, hipStream_t stream) {
    const ScoreParams sp = score_params(a.scale, a.cap);
    const int64_t rows = a.batch * a.heads * a.queries, cols = a.batch * a.kv_heads * a.keys;
    if (rows) grad_q<T, CAP><<<dim3((unsigned)((rows + 3) / 4)), kBlock, 0, stream>>>(a, sp, (float*)ws);
    if (cols) grad_kv<T, CAP><<<dim3((unsigned)((cols + 3) / 4)), kBlock, 0, stream>>>(a, sp, (const float*)ws);
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "attention gradient launch: %s", hipGetErrorString(e));
}

}  // namespace

int64_t attend_bwd_ws(const frog_attend_t& a) { return a.batch * a.heads * a.queries * 4; }

int launch_attend_bwd(const frog_attend_t& a, void* ws, hipStream_t stream) {
    if (a.type == FROG_STORAGE_F32) return a.cap > 0.f ? run<float, true>(a, ws, stream) : run<float, false>(a, ws, stream);
    if (a.type == FROG_STORAGE_F16) return a.cap > 0.f ? run<f16_t, true>(a, ws, stream) : run<f16_t, false>(a, ws, stream);
    return a.cap > 0.f ? run<bf16_t, true>(a, ws, stream) : run<bf16_t, false>(a, ws, stream);
}

}  // namespace frog

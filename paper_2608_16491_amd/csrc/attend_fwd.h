// Range attention, forward kernels (instantiated per row type by attend_*.hip).
#pragma once

#include "attend_tile.h"

namespace frog {

// Partial results of a pass split along the keys (o: null when the pass writes
// its outputs itself): part s of query row i of (sequence, kv head) x: maximum
// and sum at ml[(s * total + x * rows + i)], unnormalised output of D floats
// at o[...] (total = rows of all)
struct Parts {
    float* o;
    float2* ml;
    int64_t total;
    int splits;
};

constexpr float kLow = -FLT_MAX;   // running maximum of a row that has seen no key

// One workgroup of W wavefronts, 32 query rows each, over the keys of their
// intervals in tiles of N: scores transposed (keys x queries) so that a lane
// owns a query, one pass with the running maximum and sum, keys and values
// double buffered in LDS by direct loads.  Bound by the matrix cores and the
// exponentials beside them, two wavefronts a SIMD: 1,000 to 1,070 TFLOP/s at 8,192
// tokens, 16 heads, d = 128, bf16, every key seen (534 to 551 us); a cap costs 1.2
// to 1.4 times the time (three transcendentals a score instead of one).  fp32: 118
// TFLOP/s at 4,096 tokens.  Documents of unequal lengths leave a SIMD 1.0 to 1.3
// wavefronts on average, which is what they are bound by.
//   Weights of 16-bit rows are rounded to the type as factors of the second
// product (relative to the running maximum, so at most 2^8); their sum is of the
// 32-bit ones.  Exact to 32 bits they would be two factors, 1.5 times the
// products.  It takes the output from 0.0016 of its norm off (rounded once) to
// 0.0021 in bf16.  kAny of d = 128 spills 9 registers.
template <typename T, int D, Scores KIND, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1)))
void attend_tile(frog_attend_t a, ScoreParams sp, int group, int tiles, Parts parts, const int* order) {
    constexpr bool PLAIN = KIND == kPlain;
    constexpr int N = sizeof(T) == 2 ? 64 : 32, S = N / 32, K = D / 16, M = D / 32;
    // (buffers by name: the compiler then knows that reads of one need not wait
    // for the direct loads into the other)
    __shared__ __attribute__((aligned(16))) T k0[N * D], k1[N * D], v0[N * D], v1[N * D];
    __shared__ __attribute__((aligned(16))) float a0[64], a1[64];
    __shared__ int ends[4 * W];
    __shared__ Gaps<32 * W> rows_of;
    using L = Tile<T, D>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // heads fastest (XCDs take workgroups in turn: with 8 heads or a multiple
    // each XCD's L2 holds its own)
    const int hk = (int)(blockIdx.x % (uint32_t)a.kv_heads);
    const uint32_t rest = blockIdx.x / (uint32_t)a.kv_heads;
    const Work work(order, rest, a.batch, tiles, parts.splits);
    const int tile = work.tile, split = work.part;
    const int64_t b = work.b, x = b * a.kv_heads + hk;
    const int64_t rows = a.queries * group, row = ((int64_t)tile * W + w) * 32 + (lane & 31);
    const QueryRow q(min(row, rows - 1), group, hk);
    int lo, hi;
    interval(a, b, q.token, &lo, &hi);
    const bool some = row < rows && lo <= hi;
    // first and last key of the workgroup; of the wavefront; and the keys all its rows see
    const int wlo = col_min(some ? lo : INT_MAX), whi = col_max(some ? hi : -1);
    const int flo = col_max(some ? lo : 0), fhi = col_min(some ? hi : INT_MAX);
    if (lane == 0) {
        ends[w] = wlo;
        ends[W + w] = whi;
        ends[2 * W + w] = flo;
        ends[3 * W + w] = fhi;
    }
    if (lane < 32) {
        rows_of.lo[32 * w + lane] = some ? lo : 1;
        rows_of.hi[32 * w + lane] = some ? hi : 0;
    }
    __syncthreads();
    int first = INT_MAX, last = -1, inner_lo = 0, inner_hi = INT_MAX;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        first = min(first, ends[i]);
        last = max(last, ends[W + i]);
        inner_lo = max(inner_lo, ends[2 * W + i]);
        inner_hi = min(inner_hi, ends[3 * W + i]);
    }
    // (intervals that share a key leave no gap)
    const bool gaps = inner_lo > inner_hi && rows_of.any(last, lane);
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    if (parts.splits > 1 && last >= 0) {
        const int each = ((last - first) / parts.splits / N + 1) * N;
        const int64_t from = first + (int64_t)split * each;
        last = (int)min((int64_t)last, from + each - 1);
        first = (int)min(from, (int64_t)last + 1);
    }
    const T* kp = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2];
    const T* vp = (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2];
    const float* akp = nullptr;
    float slope = 0.f, aq = 0.f;
    if (biased<KIND>(a.slopes)) {
        akp = a.at_k + b * a.at_k_stride[0] + hk * a.at_k_stride[1];
        slope = a.slopes[q.head] * kLog2e;
        aq = a.at_q[b * a.at_q_stride + q.token];
    }
    frag<T> qf[K];
    {
        const T* p = (const T*)a.q + b * a.q_stride[0] + q.token * a.q_stride[1] + q.head * a.q_stride[2] + (lane >> 5) * 8;
#pragma unroll
        for (int s = 0; s < K; ++s) qf[s] = load_frag(p + 16 * s);
    }
    acc16 o[M];
#pragma unroll
    for (int m = 0; m < M; ++m) o[m] = acc16{};
    float top = kLow, sum = 0.f;

    auto fetch = [&](T* ks, T* vs, float* as, int j) {
        L::template load<N, W>(ks, kp, a.k_stride[1], j, last, w, lane);
        L::template load<N, W>(vs, vp, a.v_stride[1], j, last, w, lane);
        if (biased<KIND>(akp) && w == 0)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(akp + min(j + lane, last)),
                                             (__attribute__((address_space(3))) void*)as, 4, 0, 0);
    };
    auto step = [&](const T* ks, const T* vs, const float* as, int j) __attribute__((always_inline)) {
        if (j > whi || j + N <= wlo) return;
        acc16 z[S];
#pragma unroll
        for (int n = 0; n < S; ++n) {
            z[n] = acc16{};
#pragma unroll
            for (int s = 0; s < K; ++s) z[n] = mma(L::rows(ks, 32 * n, s, lane), qf[s], z[n]);
        }
        if constexpr (!PLAIN) {
            if (capped<KIND>(sp)) {
#pragma unroll
                for (int n = 0; n < S; ++n) {
                    if constexpr (KIND == kCapped) cap_shares<16>(sp, z[n]);
                    else cap_scores<16>(sp, z[n]);
                }
            } else {
#pragma unroll
                for (int n = 0; n < S; ++n) z[n] *= sp.mul;
            }
            if (biased<KIND>(akp)) {
#pragma unroll
                for (int n = 0; n < S; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const vec<float, 4> ak = *(const vec<float, 4>*)(as + 32 * n + 8 * i + 4 * (lane >> 5));
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[n][4 * i + e] = fmaf(-slope, fabsf(aq - ak[e]), z[n][4 * i + e]);
                    }
            }
        }
        if (j < flo || j + N - 1 > fhi) mask_scores<S>(z, lo - j, hi - j, lane, KIND == kCapped ? INFINITY : -INFINITY);
        float mx = z[0][0];
#pragma unroll
        for (int n = 0; n < S; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = KIND == kCapped ? fminf(mx, z[n][r]) : fmaxf(mx, z[n][r]);
        mx = half_max(PLAIN ? mx * sp.mul : KIND == kCapped ? fmaf(mx, -2.f * sp.cap2, sp.cap2) : mx);
        // the sums are scaled anew only when a row's maximum has grown by more
        // than 2^8: weights up to 256 keep their precision in every type
        if (__any(mx > top + 8.f)) {
            const float up = fmaxf(top, mx), f = exp2_fast(top - up);
            top = up;
            sum *= f;
#pragma unroll
            for (int m = 0; m < M; ++m) o[m] *= f;
        }
        const float mul = KIND == kCapped ? -2.f * sp.cap2 : sp.mul, add = KIND == kCapped ? sp.cap2 - top : -top;
#pragma unroll
        for (int n = 0; n < S; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                z[n][r] = exp2_fast(PLAIN || KIND == kCapped ? fmaf(z[n][r], mul, add) : z[n][r] - top);
                sum += z[n][r];
            }
#pragma unroll
        for (int n = 0; n < S; ++n)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const frag<T> p = to_frag<T>(z[n], t);
#pragma unroll
                for (int m = 0; m < M; ++m) o[m] = mma(L::cols(vs, 32 * n + 16 * t, m, lane), p, o[m]);
            }
    };
    // barrier: the tile has arrived in LDS, and the other buffer is read no more
    auto ready = [&] {
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0): this wavefront's own loads
        __syncthreads();
    };
    auto turn = [&](T* ks, T* vs, float* as, T* kn, T* vn, float* an, int j) {
        ready();
        if (j + N <= last) fetch(kn, vn, an, j + N);
        if (gaps) {
            rows_of.template clear<N, D, W>(vs, j, w, lane);
            __syncthreads();
        }
        step(ks, vs, as, j);
    };
    if (first <= last) {
        fetch(k0, v0, a0, first);
        for (int j = first; j <= last; j += 2 * N) {
            turn(k0, v0, a0, k1, v1, a1, j);
            if (j + N > last) break;
            turn(k1, v1, a1, k0, v0, a0, j + N);
        }
    }
    sum = half_sum(sum);
    if (row >= rows) return;
    if (!some) {
        sum = 0.f;
        top = kLow;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (parts.o) {
        const int64_t at = split * parts.total + x * rows + row;
        if (lane < 32) parts.ml[at] = make_float2(top, sum);
        if (sum > 0.f) {
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(vec<float, 4>*)(parts.o + at * D + 32 * m + 8 * i + 4 * (lane >> 5)) =
                        vec<float, 4>{o[m][4 * i], o[m][4 * i + 1], o[m][4 * i + 2], o[m][4 * i + 3]};
        }
        return;
    }
    const int64_t to = b * a.out_stride[0] + q.token * a.out_stride[1] + q.head * a.out_stride[2] + 4 * (lane >> 5);
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vec<T, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = sum > 0.f ? (T)(o[m][4 * i + e] * inv) : (T)0.f;
            *(vec<T, 4>*)((T*)a.out + to + 32 * m + 8 * i) = y;
        }
    if (sizeof(T) == 2 && a.out_low) {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vec<T, 4> y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = sum > 0.f ? rounded_off<T>(o[m][4 * i + e] * inv) : (T)0.f;
                *(vec<T, 4>*)((T*)a.out_low + to + 32 * m + 8 * i) = y;
            }
    }
    if (a.lse && lane < 32) a.lse[(b * a.heads + q.head) * a.queries + q.token] = sum > 0.f ? (top + __log2f(sum)) * kLn2 : -INFINITY;
}

// Keys of one sequence and kv head, in one piece or in pages.
template <typename T>
struct FlatKeys {
    const T *k, *v;
    int64_t ks, vs;
    struct Where {
        int j;
    };
    __device__ inline Where where(int j) const { return {j}; }
    // row i (0 .. 31) of the 32 whose Where the lanes hold
    __device__ static inline Where of(Where x, int i, int j, int last) { return {min(j + i, last)}; }
    __device__ inline const T* key(Where x) const { return k + x.j * ks; }
    __device__ inline const T* value(Where x) const { return v + x.j * vs; }
    static constexpr bool kPaged = false;
    __device__ static inline bool real(Where) { return true; }
};

template <typename T>
struct PagedKeys {
    const T *k, *v;          // at the kv head
    int64_t ks[2], vs[2];    // page, row
    const int32_t* pages;    // of the request
    uint32_t page;
    int64_t num_pages;
    const T* spare;          // D values that may be read, for rows without a page
    struct Where {
        int page, row;       // page -1: no such page
    };
    __device__ inline Where where(int j) const {
        const uint32_t p = (uint32_t)j / page;
        const int at = pages[p];
        return {at >= 0 && at < num_pages ? at : -1, (int)((uint32_t)j - p * page)};
    }
    __device__ static inline Where of(Where x, int i, int, int) { return {__shfl(x.page, i), __shfl(x.row, i)}; }
    __device__ inline const T* key(Where x) const { return x.page >= 0 ? k + x.page * ks[0] + x.row * ks[1] : spare; }
    __device__ inline const T* value(Where x) const { return x.page >= 0 ? v + x.page * vs[0] + x.row * vs[1] : spare; }
    static constexpr bool kPaged = true;
    __device__ static inline bool real(Where x) { return x.page >= 0; }
};

// The query rows of a wavefront's few-rows pass: column lane % 16 of each of
// the RG groups of 16.
template <int RG>
struct FewRows {
    int lo[RG], hi[RG];       // interval (lo > hi: no row, or an empty one)
    float slope[RG], aq[RG];  // distance bias
    float top[RG], sum[RG];
};

// Few query rows (at most 16 RG, a token's group of heads after another) over
// the keys first..last of one (sequence, kv head), 32 keys a step and
// wavefront, wavefront w of W taking every W-th step.  Nothing passes through
// LDS: a lane loads 16 bytes of a key row as it stands in the left factor of
// the scores, and D / 16 values each of 8 value rows, whose transposition is
// a renaming of registers and one exchange of 16-bit halves; the output's
// columns come out as d = 4 (L/16) + r times D/16 plus e.  Weights of 16-bit rows
// are two factors of the second product, the rounded weight and what that left:
// beside the reads of the cache the second product is nearly free (1,001 keys 13.7
// -> 13.9 us, 16 caches to 10,000 unchanged), and the output's only rounding is its own.
template <typename T, int D, int RG>
struct FewPass {
    static constexpr int K = D / 32, C = D / 16;
    frag<T> q[RG][K];
    acc4 o[RG][C];
    FewRows<RG> row;

    __device__ inline void reset() {
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            row.top[g] = kLow;
            row.sum[g] = 0.f;
#pragma unroll
            for (int e = 0; e < C; ++e) o[g][e] = acc4{};
        }
    }

    // PLAIN: neither cap nor bias.  at_key(j): attribute of key j (with a bias);
    // store(g, j, z, whole): takes four scores of the keys from j in log2 units
    // (whole: all of them exist).
    // The next step's keys are loaded once the scores have been taken from
    // this one's registers, its values after the second product: two loads
    // are in flight behind the arithmetic without registers for a second step.
    template <bool PLAIN, typename Keys, typename At, typename Store>
    __device__ inline void run(const Keys& keys, const ScoreParams& sp, bool bias, At&& at_key, Store&& store, int first, int last, int w,
                               int W, int lane) {
        const int c = lane & 15, h = lane >> 4;
        int fit_lo = 0, fit_hi = last;   // keys every real row sees
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            const bool some = row.lo[g] <= row.hi[g];
            fit_lo = max(fit_lo, col_max(some ? row.lo[g] : 0));
            fit_hi = min(fit_hi, col_min(some ? row.hi[g] : INT_MAX));
        }
        frag<T> kf[2][K];   // key rows c and 16 + c
        vec<T, C> vv[8];    // value rows 4h .. 4h+3 and 16 + 4h ..
        uint32_t real = 255, coming = 255;   // bit e: value row e has a page
        typename Keys::Where mine{};
        auto row_of = [&](int e) { return 16 * (e >> 2) + 4 * h + (e & 3); };
        auto load_keys = [&](int j) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const T* p = keys.key(Keys::of(mine, 16 * u + c, j, last)) + 8 * h;
#pragma unroll
                for (int s = 0; s < K; ++s) kf[u][s] = load_frag(p + 32 * s);
            }
        };
        auto load_values = [&](int j) {
            if (Keys::kPaged) coming = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const auto at = Keys::of(mine, row_of(e), j, last);
                vv[e] = load_piece<T, C>(keys.value(at) + C * c);
                if (Keys::kPaged) coming |= (uint32_t)Keys::real(at) << e;
            }
        };
        int64_t j64 = (int64_t)first + 32 * w;
        if (j64 > last) return;
        mine = keys.where((int)min(j64 + (lane & 31), (int64_t)last));
        load_keys((int)j64);
        load_values((int)j64);
        real = coming;
        auto step = [&](auto masked, int j, bool more, int next) __attribute__((always_inline)) {
            constexpr bool MASKED = decltype(masked)::value;
            if (more) mine = keys.where((int)min((int64_t)next + (lane & 31), (int64_t)last));
            float z[RG][8];
#pragma unroll
            for (int g = 0; g < RG; ++g)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    acc4 s4 = acc4{};
#pragma unroll
                    for (int s = 0; s < K; ++s) s4 = mma(kf[u][s], q[g][s], s4);
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[g][4 * u + r] = s4[r];
                }
            if (more) load_keys(next);
            float ak[8];
            if (!PLAIN && bias) {
#pragma unroll
                for (int e = 0; e < 8; ++e) ak[e] = at_key(min(j + row_of(e), last));
            }
            uint32_t met = 0;
            frag<T> p[RG], low[RG];
#pragma unroll
            for (int g = 0; g < RG; ++g) {
                if (!PLAIN && sp.cap2 > 0.f) {
                    cap_scores<8>(sp, z[g]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[g][e] *= sp.mul;
                }
                if (!PLAIN && bias) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[g][e] = fmaf(-row.slope[g], fabsf(row.aq[g] - ak[e]), z[g][e]);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) store(g, j + row_of(4 * u), &z[g][4 * u], !MASKED);
                if constexpr (MASKED) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int at = j + row_of(e);
                        const bool in = at >= row.lo[g] && at <= min(row.hi[g], last) && ((real >> e) & 1);
                        z[g][e] = in ? z[g][e] : -INFINITY;
                        met |= (uint32_t)(((__ballot(in) >> (16 * h)) & 0xffff) != 0) << e;
                    }
                }
                float mx = z[g][0];
#pragma unroll
                for (int e = 1; e < 8; ++e) mx = fmaxf(mx, z[g][e]);
                mx = quarter_max(mx);
                if (__any(mx > row.top[g] + 8.f)) {
                    const float up = fmaxf(row.top[g], mx), f = exp2_fast(row.top[g] - up);
                    row.top[g] = up;
                    row.sum[g] *= f;
#pragma unroll
                    for (int e = 0; e < C; ++e) o[g][e] *= f;
                }
                vec<float, 8> y;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = exp2_fast(z[g][e] - row.top[g]);
                    row.sum[g] += y[e];
                }
                if constexpr (sizeof(T) == 4) {
                    p[g] = y;
                } else {
                    p[g] = __builtin_convertvector(y, frag<T>);
                    low[g] = __builtin_convertvector(y - __builtin_convertvector(p[g], vec<float, 8>), frag<T>);
                }
            }
            if constexpr (MASKED) {
                // values of keys that no row sees may be anything, and must not
                // meet a weight of 0 in the second product
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!((met >> e) & 1)) vv[e] = vec<T, C>{};
            }
#pragma unroll
            for (int e = 0; e < C; ++e) {
                const frag<T> vf{vv[0][e], vv[1][e], vv[2][e], vv[3][e], vv[4][e], vv[5][e], vv[6][e], vv[7][e]};
#pragma unroll
                for (int g = 0; g < RG; ++g) {
                    o[g][e] = mma(vf, p[g], o[g][e]);
                    if constexpr (sizeof(T) == 2) o[g][e] = mma(vf, low[g], o[g][e]);
                }
            }
            if (more) {
                load_values(next);
                real = coming;
            }
        };
        for (;;) {
            const int j = (int)j64;
            const int64_t next = j64 + 32 * W;
            const bool more = next <= last;
            if (j >= fit_lo && j + 31 <= fit_hi && (!Keys::kPaged || __all(real == 255))) step(std::false_type{}, j, more, (int)min(next, (int64_t)last));
            else step(std::true_type{}, j, more, (int)min(next, (int64_t)last));
            if (!more) break;
            j64 = next;
        }
    }

    // Joins the W wavefronts' results: pairs of halves, through LDS in the
    // registers' own layout, then the rows of the whole in lds (16 RG of D + 4
    // floats, unnormalised) and their maxima and sums in tops, sums (W RG 16
    // floats each).  Starts and ends with a barrier.
    static constexpr int kJoin(int W) { return (W / 2) * 64 * RG * C * 4 > 16 * RG * (D + 4) ? (W / 2) * 64 * RG * C * 4 : 16 * RG * (D + 4); }
    template <int W>
    __device__ inline void join(float* lds, float* tops, float* sums, int w, int lane) {
        const int c = lane & 15, h = lane >> 4;
#pragma unroll
        for (int g = 0; g < RG; ++g) row.sum[g] = quarter_sum(row.sum[g]);
#pragma unroll
        for (int g = 0; g < RG; ++g)
            if (h == 0) {
                tops[(w * RG + g) * 16 + c] = row.top[g];
                sums[(w * RG + g) * 16 + c] = row.sum[g];
            }
        __syncthreads();
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            float top = kLow, sum = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) top = fmaxf(top, tops[(i * RG + g) * 16 + c]);
#pragma unroll
            for (int i = 0; i < W; ++i) sum += sums[(i * RG + g) * 16 + c] * exp2_fast(tops[(i * RG + g) * 16 + c] - top);
            const float f = exp2_fast(row.top[g] - top);
#pragma unroll
            for (int e = 0; e < C; ++e) o[g][e] *= f;
            row.top[g] = top;
            row.sum[g] = sum;
        }
        acc4* slots = (acc4*)lds;
#pragma unroll
        for (int half = W / 2; half >= 1; half /= 2) {
            if (w >= half && w < 2 * half) {
#pragma unroll
                for (int g = 0; g < RG; ++g)
#pragma unroll
                    for (int e = 0; e < C; ++e) slots[((w - half) * RG * C + g * C + e) * 64 + lane] = o[g][e];
            }
            __syncthreads();
            if (w < half) {
#pragma unroll
                for (int g = 0; g < RG; ++g)
#pragma unroll
                    for (int e = 0; e < C; ++e) o[g][e] += slots[(w * RG * C + g * C + e) * 64 + lane];
            }
            __syncthreads();
        }
        if (w == 0) {
#pragma unroll
            for (int g = 0; g < RG; ++g) {
                if (h == 0) {
                    tops[16 * g + c] = row.top[g];
                    sums[16 * g + c] = row.lo[g] <= row.hi[g] ? row.sum[g] : 0.f;
                }
#pragma unroll
                for (int e = 0; e < C; ++e)
#pragma unroll
                    for (int r = 0; r < 4; ++r) lds[(16 * g + c) * (D + 4) + (4 * h + r) * C + e] = o[g][e][r];
            }
        }
        __syncthreads();
    }
};

// One workgroup per (sequence, kv head, part of the keys) for at most 16 RG
// query rows.  Bound by HBM, 4.4 TB/s over 24 caches to 40,000 keys of 8 kv heads
// (443 us), fp32 5.8 over 16 of 10,000; a short cache by its chain of steps (1,001
// keys 13.4 us; split 6, and 4 for the join).  fp32 rows of d = 128 spill 16 to 45 registers
// in two groups (8 caches of 10,000, 2 kv heads of 32: 78 us, 2.1 TB/s; bf16 45, 1.8).
// KEEP: scores [batch][heads][queries][keys] receive every score in log2 units
// for the key weights.
template <typename T, int D, int RG, int W, bool PLAIN, bool KEEP>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(RG == 1 && sizeof(T) == 2 ? 2 : 1))) void attend_few(frog_attend_t a, ScoreParams sp, int group, Parts parts, float* scores) {
    __shared__ __attribute__((aligned(16))) float lds[FewPass<T, D, RG>::kJoin(W)], tops[W * RG * 16], sums[W * RG * 16];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t pairs = (uint32_t)(a.batch * a.kv_heads), x = blockIdx.x % pairs;
    const int split = (int)(blockIdx.x / pairs);
    const int64_t b = x / (uint32_t)a.kv_heads;
    const int hk = (int)(x % (uint32_t)a.kv_heads), rows = (int)a.queries * group;
    FewPass<T, D, RG> f;
    f.reset();
    int first = INT_MAX, last = -1;
    float* zp[RG];
#pragma unroll
    for (int g = 0; g < RG; ++g) {
        const int r = 16 * g + (lane & 15);
        const QueryRow q(min(r, rows - 1), group, hk);
        int lo, hi;
        interval(a, b, q.token, &lo, &hi);
        if (r >= rows) lo = 0, hi = -1;
        f.row.lo[g] = lo;
        f.row.hi[g] = hi;
        first = min(first, col_min(lo <= hi ? lo : INT_MAX));
        last = max(last, col_max(lo <= hi ? hi : -1));
        f.row.slope[g] = a.slopes ? a.slopes[q.head] * kLog2e : 0.f;
        f.row.aq[g] = a.slopes ? a.at_q[b * a.at_q_stride + q.token] : 0.f;
        zp[g] = KEEP && r < rows ? scores + ((b * a.heads + q.head) * a.queries + q.token) * a.keys : nullptr;
        const T* p = (const T*)a.q + b * a.q_stride[0] + q.token * a.q_stride[1] + q.head * a.q_stride[2] + (lane >> 4) * 8;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) f.q[g][s] = load_frag(p + 32 * s);
    }
    if (parts.splits > 1 && last >= 0) {
        const int each = ((last - first) / parts.splits / (32 * W) + 1) * (32 * W);
        const int64_t from = first + (int64_t)split * each;
        last = (int)min((int64_t)last, from + each - 1);
        first = (int)min(from, (int64_t)last + 1);
    }
    const FlatKeys<T> keys{(const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2], (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2],
                           a.k_stride[1], a.v_stride[1]};
    const float* akp = a.slopes ? a.at_k + b * a.at_k_stride[0] + hk * a.at_k_stride[1] : nullptr;
    if (first <= last)
        f.template run<PLAIN>(keys, sp, akp != nullptr, [&](int j) { return akp[j]; },
                              [&](int g, int j, const float* z, bool all) {
                                  if (!KEEP || !zp[g]) return;
                                  using f4 = float __attribute__((ext_vector_type(4), aligned(4)));
                                  if (all) *(f4*)(zp[g] + j) = f4{z[0], z[1], z[2], z[3]};
                                  else
                                      for (int e = 0; e < 4; ++e)
                                          if (j + e <= last) zp[g][j + e] = z[e];
                              },
                              first, last, w, W, lane);
    f.template join<W>(lds, tops, sums, w, lane);
    // joint rows: out, or this part's
    for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * W) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        const float sum = sums[r], inv = sum > 0.f ? 1.f / sum : 0.f;
        const acc4 y = *(const acc4*)(lds + r * (D + 4) + d);
        if (parts.o) {
            const int64_t at = split * parts.total + (int64_t)x * rows + r;
            if (sum > 0.f) *(acc4*)(parts.o + at * D + d) = y;
            if (d == 0) parts.ml[at] = make_float2(tops[r], sum);
        } else {
            const QueryRow q(r, group, hk);
            const int64_t to = b * a.out_stride[0] + q.token * a.out_stride[1] + q.head * a.out_stride[2] + d;
            vec<float, 4> t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = sum > 0.f ? y[e] * inv : 0.f;
            put_rounded<T, 4>((T*)a.out + to, a.out_low ? (T*)a.out_low + to : nullptr, t);
            if (a.lse && d == 0) a.lse[(b * a.heads + q.head) * a.queries + q.token] = sum > 0.f ? (tops[r] + __log2f(sum)) * kLn2 : -INFINITY;
        }
    }
}

// One token of each of many requests over their shared prefix and their own
// tails, for few rows: workgroups below `head` take a part of the prefix for
// the rows of all requests (at most 16 RG per kv head; none when the prefix is
// left to attend_tile), the others a part of one request's tail for 16 RG rows
// of a kv head's group.  Bound by HBM and, at d = 128, by its registers (15 to 21
// spilled; fp32 in two groups 87 to 123): 100 tails to 2,000 rows, 8 kv heads, d =
// 128, bf16, 112 to 120 us (3.7 to 3.4 TB/s).
template <typename T, int D, int RG, bool PLAIN>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RG == 1 && sizeof(T) == 2 ? 2 : 1))) void shared_few(frog_attend_shared_t a, ScoreParams sp, int group, int head, Parts prefix, Parts tail) {
    constexpr int W = 4;
    __shared__ __attribute__((aligned(16))) float lds[FewPass<T, D, RG>::kJoin(W)], tops[W * RG * 16], sums[W * RG * 16];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    FewPass<T, D, RG> f;
    f.reset();
    const bool own = (int)blockIdx.x >= head;    // a tail
    const int row_groups = (group + 16 * RG - 1) / (16 * RG);
    uint32_t x = own ? blockIdx.x - head : blockIdx.x;
    const int hk = (int)(x % (uint32_t)a.kv_heads);
    x /= (uint32_t)a.kv_heads;
    int row0 = 0, split;
    int64_t b = 0;
    if (own) {
        row0 = (int)(x % (uint32_t)row_groups) * 16 * RG;
        x /= (uint32_t)row_groups;
        b = x % (uint32_t)a.batch;
        split = (int)(x / (uint32_t)a.batch);
    } else {
        split = (int)x;
    }
    const Parts& parts = own ? tail : prefix;
    const int rows = own ? min(group - row0, 16 * RG) : (int)a.batch * group;
    const int64_t most = a.pages_per_request * a.page;
    int first = INT_MAX, last = -1;
#pragma unroll
    for (int g = 0; g < RG; ++g) {
        const int r = min(16 * g + (lane & 15), rows - 1);
        const int64_t req = own ? b : r / group;
        const int h = hk * group + (own ? row0 + r : r % group);
        const int len = a.pages_per_request > 0 ? (int)min((int64_t)max(a.lengths[req], 0), most) : 0;
        int lo = 0, hi = own ? len - 1 : (int)a.prefix - 1;
        if (!own && a.lr) {
            const int2 p = *(const int2*)(a.lr + 2 * req);
            lo = max(lo, p.x);
            hi = min(hi, p.y);
        }
        if (16 * g + (lane & 15) >= rows) lo = 0, hi = -1;
        f.row.lo[g] = lo;
        f.row.hi[g] = hi;
        first = min(first, col_min(lo <= hi ? lo : INT_MAX));
        last = max(last, col_max(lo <= hi ? hi : -1));
        f.row.slope[g] = a.slopes ? a.slopes[h] * kLog2e : 0.f;
        f.row.aq[g] = (float)((own ? 0 : a.prefix) + len - 1);
        const T* p = (const T*)a.q + req * a.q_stride[0] + h * a.q_stride[1] + (lane >> 4) * 8;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) f.q[g][s] = load_frag(p + 32 * s);
    }
    if (parts.splits > 1 && last >= 0) {
        const int each = ((last - first) / parts.splits / (32 * W) + 1) * (32 * W);
        const int64_t from = first + (int64_t)split * each;
        last = (int)min((int64_t)last, from + each - 1);
        first = (int)min(from, (int64_t)last + 1);
    }
    auto at_key = [](int j) { return (float)j; };
    auto none = [](int, int, const float*, bool) {};
    if (first <= last) {
        if (own) {
            const PagedKeys<T> keys{(const T*)a.k_pages + hk * a.k_pages_stride[2], (const T*)a.v_pages + hk * a.v_pages_stride[2],
                                    {a.k_pages_stride[0], a.k_pages_stride[1]}, {a.v_pages_stride[0], a.v_pages_stride[1]},
                                    a.pages + b * a.pages_per_request, (uint32_t)a.page, a.num_pages,
                                    (const T*)a.q + b * a.q_stride[0] + hk * group * a.q_stride[1]};
            f.template run<PLAIN>(keys, sp, a.slopes != nullptr, at_key, none, first, last, w, W, lane);
        } else {
            const FlatKeys<T> keys{(const T*)a.k + hk * a.k_stride[1], (const T*)a.v + hk * a.v_stride[1], a.k_stride[0], a.v_stride[0]};
            f.template run<PLAIN>(keys, sp, a.slopes != nullptr, at_key, none, first, last, w, W, lane);
        }
    }
    f.template join<W>(lds, tops, sums, w, lane);
    const int64_t base = split * parts.total + (own ? (b * a.kv_heads + hk) * group + row0 : (int64_t)hk * rows);
    for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * W) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        if (sums[r] > 0.f) *(acc4*)(parts.o + (base + r) * D + d) = *(const acc4*)(lds + r * (D + 4) + d);
        if (d == 0) parts.ml[base + r] = make_float2(tops[r], sums[r]);
    }
}

// The same where prefix and tails are short: one workgroup does both for 16 RG
// rows of a (request, kv head) and nothing is left to join (the prefix comes
// from L2 for all requests but the first).  d = 128 spills 5 to 11 registers, fp32
// in two groups 88 to 109.
template <typename T, int D, int RG, int W, bool PLAIN>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(RG == 1 && sizeof(T) == 2 ? 2 : 1))) void shared_whole(frog_attend_shared_t a, ScoreParams sp, int group) {
    __shared__ __attribute__((aligned(16))) float lds[FewPass<T, D, RG>::kJoin(W)], tops[W * RG * 16], sums[W * RG * 16];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row_groups = (group + 16 * RG - 1) / (16 * RG);
    uint32_t x = blockIdx.x;
    const int hk = (int)(x % (uint32_t)a.kv_heads);
    x /= (uint32_t)a.kv_heads;
    const int row0 = (int)(x % (uint32_t)row_groups) * 16 * RG, rows = min(group - row0, 16 * RG);
    const int64_t b = x / (uint32_t)row_groups;
    const int len = a.pages_per_request > 0 ? (int)min((int64_t)max(a.lengths[b], 0), a.pages_per_request * a.page) : 0;
    int lo = 0, hi = (int)a.prefix - 1;
    if (a.lr) {
        const int2 p = *(const int2*)(a.lr + 2 * b);
        lo = max(lo, p.x);
        hi = min(hi, p.y);
    }
    FewPass<T, D, RG> f;
    f.reset();
#pragma unroll
    for (int g = 0; g < RG; ++g) {
        const int h = hk * group + row0 + min(16 * g + (lane & 15), rows - 1);
        f.row.slope[g] = a.slopes ? a.slopes[h] * kLog2e : 0.f;
        const T* p = (const T*)a.q + b * a.q_stride[0] + h * a.q_stride[1] + (lane >> 4) * 8;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) f.q[g][s] = load_frag(p + 32 * s);
    }
    auto pass = [&](auto& keys, int first, int last, float at) {
#pragma unroll
        for (int g = 0; g < RG; ++g) {
            f.row.lo[g] = first;
            f.row.hi[g] = 16 * g + (lane & 15) < rows ? last : -1;
            f.row.aq[g] = at;
        }
        if (first <= last)
            f.template run<PLAIN>(keys, sp, a.slopes != nullptr, [](int j) { return (float)j; }, [](int, int, const float*, bool) {}, first, last, w, W, lane);
    };
    const FlatKeys<T> head{(const T*)a.k + hk * a.k_stride[1], (const T*)a.v + hk * a.v_stride[1], a.k_stride[0], a.v_stride[0]};
    pass(head, lo, hi, (float)(a.prefix + len - 1));
    const PagedKeys<T> tail{(const T*)a.k_pages + hk * a.k_pages_stride[2], (const T*)a.v_pages + hk * a.v_pages_stride[2],
                            {a.k_pages_stride[0], a.k_pages_stride[1]}, {a.v_pages_stride[0], a.v_pages_stride[1]},
                            a.pages + b * a.pages_per_request, (uint32_t)a.page, a.num_pages,
                            (const T*)a.q + b * a.q_stride[0] + hk * group * a.q_stride[1]};
    pass(tail, 0, len - 1, (float)(len - 1));
#pragma unroll
    for (int g = 0; g < RG; ++g) f.row.lo[g] = f.row.hi[g] = 0;   // (rows past the group hold sums of steps without a mask, and are not written)
    f.template join<W>(lds, tops, sums, w, lane);
    for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * W) {
        const int r = i / (D / 4), d = i % (D / 4) * 4, h = hk * group + row0 + r;
        const float sum = sums[r], inv = sum > 0.f ? 1.f / sum : 0.f;
        const acc4 y = *(const acc4*)(lds + r * (D + 4) + d);
        vec<T, 4> t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = (T)(y[e] * inv);
        *(vec<T, 4>*)((T*)a.out + b * a.out_stride[0] + h * a.out_stride[1] + d) = t;
        if (a.lse && d == 0) a.lse[b * a.heads + h] = sum > 0.f ? (tops[r] + __log2f(sum)) * kLn2 : -INFINITY;
    }
}

// The parts of one query row, joined: one wavefront, D / 64 neighbouring
// values a lane (half the lanes of D = 32 idle; D = 96 takes 1.5 as 2).
template <int D>
struct Joined {
    static constexpr int V = D > 64 ? 2 : 1;
    float y[V];
    float top, sum;
    __device__ inline Joined() : top(kLow), sum(0.f) {
        for (int v = 0; v < V; ++v) y[v] = 0.f;
    }
    // maxima and sums alone
    __device__ inline float add_sums(const Parts& p, int64_t i, int s0, int lane) {
        const float2 ml = s0 + lane < p.splits ? p.ml[(s0 + lane) * p.total + i] : make_float2(kLow, 0.f);
        float up = ml.y > 0.f ? ml.x : kLow;
        for (int o = 32; o; o >>= 1) up = fmaxf(up, __shfl_xor(up, o));
        up = fmaxf(up, top);
        const float f = exp2_fast(top - up), w = ml.y > 0.f ? exp2_fast(ml.x - up) : 0.f;
        float all = ml.y * w;
        for (int o = 32; o; o >>= 1) all += __shfl_xor(all, o);
        sum = sum * f + all;
#pragma unroll
        for (int v = 0; v < V; ++v) y[v] *= f;
        top = up;
        return w;
    }
    __device__ inline void add(const Parts& p, int64_t i, int lane) {
        const int d = min(lane * V, D - V);
        for (int s0 = 0; s0 < p.splits; s0 += 64) {
            const float w = add_sums(p, i, s0, lane);
            const int n = min(64, p.splits - s0);
            const float* o = p.o + (s0 * p.total + i) * D + d;
            // eight parts' reads in flight; a part without a key is not
            // written, and may hold anything
            for (int s = 0; s < n; s += 8) {
                vec<float, V> x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = *(const vec<float, V>*)(o + min(s + u, n - 1) * p.total * D);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const float ws = __shfl(w, (s + u) & 63);
                    if (s + u < n && ws > 0.f) {
#pragma unroll
                        for (int v = 0; v < V; ++v) y[v] = fmaf(ws, x[u][v], y[v]);
                    }
                }
            }
        }
    }
    template <typename T>
    __device__ inline void write(T* out, T* low, int lane) const {
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        if (lane * V >= D) return;
        vec<float, V> t;
#pragma unroll
        for (int v = 0; v < V; ++v) t[v] = y[v] * inv;
        put_rounded<T, V>(out + lane * V, low ? low + lane * V : nullptr, t);
    }
    __device__ inline float lse() const { return sum > 0.f ? (top + __log2f(sum)) * kLn2 : -INFINITY; }
};

template <typename T, int D>
__device__ inline void join_row(const frog_attend_t& a, int group, const Parts& parts, int64_t i, int lane) {
    const int64_t rows = a.queries * group;
    if (i >= parts.total) return;
    const int64_t x = i / rows, b = x / a.kv_heads;
    const QueryRow q(i % rows, group, (int)(x % a.kv_heads));
    Joined<D> y;
    y.add(parts, i, lane);
    const int64_t to = b * a.out_stride[0] + q.token * a.out_stride[1] + q.head * a.out_stride[2];
    y.write((T*)a.out + to, a.out_low ? (T*)a.out_low + to : nullptr, lane);
    if (a.lse && lane == 0) a.lse[(b * a.heads + q.head) * a.queries + q.token] = y.lse();
}

template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join(frog_attend_t a, int group, Parts parts) {
    join_row<T, D>(a, group, parts, (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), threadIdx.x & 63);
}

// The end of a few-rows pass that wants key weights: the first `joins`
// workgroups join its parts (none where it was not split), the others take
// 256 keys of a (sequence, kv head) each, from the scores the pass kept and
// the parts' maxima and sums.
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_few_end(frog_attend_t a, int group, Parts parts, const float* scores, int joins) {
    __shared__ float lse2[32];
    __shared__ int lo[32], hi[32];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    if ((int)blockIdx.x < joins) {
        join_row<T, D>(a, group, parts, (int64_t)blockIdx.x * 4 + w, lane);
        return;
    }
    const uint32_t at = blockIdx.x - joins, pairs = (uint32_t)(a.batch * a.kv_heads), x = at % pairs;
    const int64_t b = x / (uint32_t)a.kv_heads, j = (int64_t)(at / pairs) * 256 + threadIdx.x;
    const int hk = (int)(x % (uint32_t)a.kv_heads), rows = (int)a.queries * group;
    for (int r = w; r < rows; r += 4) {
        const QueryRow q(r, group, hk);
        float z;
        if (joins) {
            Joined<D> y;
            for (int s = 0; s < parts.splits; s += 64) y.add_sums(parts, (int64_t)x * rows + r, s, lane);
            z = y.sum > 0.f ? y.top + __log2f(y.sum) : INFINITY;
        } else {
            z = a.lse[(b * a.heads + q.head) * a.queries + q.token] * kLog2e;
            if (z == -INFINITY) z = INFINITY;
        }
        if (lane == 0) {
            lse2[r] = z;
            interval(a, b, q.token, &lo[r], &hi[r]);
        }
    }
    __syncthreads();
    if (j >= a.keys) return;
    float sum = 0.f;
    for (int r0 = 0; r0 < rows; r0 += 4) {
        float z[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const QueryRow q(min(r0 + u, rows - 1), group, hk);
            z[u] = scores[((b * a.heads + q.head) * a.queries + q.token) * a.keys + j];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int r = min(r0 + u, rows - 1);
            if (r0 + u < rows && j >= lo[r] && j <= hi[r]) sum += weight2(z[u] - lse2[r]);
        }
    }
    const int64_t i = (int64_t)x * a.keys + j;
    a.w_out[i] = (a.w_in ? a.w_in[i] : 0.f) + sum;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void shared_join(frog_attend_shared_t a, int group, Parts prefix, Parts tail) {
    const int lane = threadIdx.x & 63;
    const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= a.batch * a.heads) return;
    const int64_t b = i / a.heads;
    const int h = (int)(i % a.heads);
    Joined<D> y;
    y.add(prefix, (h / group * a.batch + b) * group + h % group, lane);
    y.add(tail, i, lane);
    y.write((T*)a.out + b * a.out_stride[0] + h * a.out_stride[1], (T*)nullptr, lane);
    if (a.lse && lane == 0) a.lse[i] = y.lse();
}

// The attributes of a biased pass over a shared prefix: keys stand at their
// numbers, request b's query at prefix + its tail's length - 1.
static __global__ __launch_bounds__(256) void shared_places(frog_attend_shared_t a, float* at_q, float* at_k) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < a.prefix) at_k[i] = (float)i;
    if (i >= a.batch) return;
    const int64_t len = a.pages_per_request > 0 ? min((int64_t)max(a.lengths[i], 0), a.pages_per_request * a.page) : 0;
    at_q[i] = (float)(a.prefix + len - 1);
}

}  // namespace frog

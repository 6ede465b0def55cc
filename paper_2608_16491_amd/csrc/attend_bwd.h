// Range attention, gradients and key weights (instantiated per row type by
// attend_*.hip).
#pragma once

#include "attend_tile.h"

namespace frog {

// What the passes that own keys need of 32 query rows at a time, prepared once
// per call: per (sequence, kv head) and tile of 32 rows a block of floats
// (lse in log2 units, less capL for kCapped, +inf for a row without keys; delta = dout . out; the
// interval, as integers; bias slope and attribute), per (sequence, tile) the
// least and largest key of the rows' intervals, and the keys all of them see
// (z > w when a row has none), and a row of zeros that stands for the rows
// without keys, whose memory may hold anything.
struct RowPack {
    static constexpr int kLse = 0, kDelta = 32, kLo = 64, kHi = 96, kSlope = 128, kAt = 160, kFloats = 192;
    float* rows;       // [batch * kv_heads][tiles][kFloats]
    int4* bounds;      // [batch][tiles]
    void* zeros;       // 512 bytes
    int tiles;
};

// delta is a 32-bit sum over the output and what its rounding left (out_low).
// Where a row's weight lies on few keys, dout . v - delta is small beside both: from
// the rounded output alone dq and dk of 16-bit causal rows were off by 2.7 times a
// single rounding at 2 tokens, 1.7 at 64 and 1.5 at 2,500 (1.41, the square root of
// 2, is what rounding dx leaves).  The output itself is a sum of rounded weights,
// which few keys do not average out (still 1.53 at 2 tokens): of 16-bit rows that
// see at most kSummedKeys keys delta is sum p (dout . v), by its definition.
// 8,192 tokens, 16 heads, d = 128, bf16: 18 us (100 MB), 23 where a wavefront has
// such rows (26 with the tiles of one kv head after another).
constexpr int kSummedKeys = 16;
template <typename T, int D, bool GRAD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void pack_rows(frog_attend_t a, ScoreParams sp, int group, RowPack pack, const float* lse, float shift) {
    const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
    if (blockIdx.x == 0 && threadIdx.x < 128) ((float*)pack.zeros)[threadIdx.x] = 0.f;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), pairs = a.batch * a.kv_heads;
    if (at >= pairs * pack.tiles) return;
    // (earlier tiles first: there the rows stand that take longest, see below)
    const int64_t x = at % pairs, b = x / a.kv_heads;
    const int tile = (int)(at / pairs), hk = (int)(x % a.kv_heads);
    const int64_t rows = a.queries * group, row = (int64_t)tile * 32 + i;
    const QueryRow q(min(row, rows - 1), group, hk);
    int lo, hi;
    interval(a, b, q.token, &lo, &hi);
    const bool some = row < rows && lo <= hi;
    if (!some) lo = 1, hi = 0;
    float* out = pack.rows + (x * pack.tiles + tile) * RowPack::kFloats;
    const int64_t stat = (b * a.heads + q.head) * a.queries + q.token;
    // (-inf: no key, or a bias that leaves none a weight)
    const float lse2 = some && lse[stat] > -INFINITY ? lse[stat] * kLog2e : INFINITY;
    if constexpr (GRAD) {
        // a piece of 16 bytes a lane, LANES lanes a row (a power of two; D = 96
        // leaves some without one), as many rows at once as fit
        constexpr int PER = 16 / sizeof(T), PIECES = D / PER, LANES = PIECES <= 4 ? 4 : PIECES <= 8 ? 8 : PIECES <= 16 ? 16 : 32, AT = 64 / LANES;
        const int piece = lane % LANES;
        const bool few = sizeof(T) == 2 && some && hi - lo < kSummedKeys;
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += AT) {
            const int r = r0 + lane / LANES;
            const QueryRow qr(min((int64_t)tile * 32 + r, rows - 1), group, hk);
            float delta = 0.f;
            if (piece < PIECES) {
                const vec<T, PER> u = *(const vec<T, PER>*)((const T*)a.dout + b * a.dout_stride[0] + qr.token * a.dout_stride[1] +
                                                            qr.head * a.dout_stride[2] + piece * PER);
                const int64_t at_out = b * a.out_stride[0] + qr.token * a.out_stride[1] + qr.head * a.out_stride[2] + piece * PER;
                const vec<T, PER> v = *(const vec<T, PER>*)((const T*)a.out + at_out);
#pragma unroll
                for (int e = 0; e < PER; ++e) delta = fmaf((float)u[e], (float)v[e], delta);
                if (sizeof(T) == 2 && a.out_low) {
                    const vec<T, PER> low = *(const vec<T, PER>*)((const T*)a.out_low + at_out);
#pragma unroll
                    for (int e = 0; e < PER; ++e) delta = fmaf((float)u[e], (float)low[e], delta);
                }
            }
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) delta += __shfl_xor(delta, o);
            const int state = __shfl(few ? 2 : some ? 1 : 0, r);   // row r's lane
            if (piece == 0 && state < 2) out[RowPack::kDelta + r] = state ? delta : 0.f;
        }
        if constexpr (sizeof(T) == 2) {
            // the others, from the least of their keys on 32 at a time, as in
            // attend_keys: a lane owns a row, so the sums stay in it
            float delta = 0.f;
            for (bool left = few; __any(left);) {
                const int first = col_min(left ? lo : INT_MAX), j = min(first + i, (int)a.keys - 1);
                const T* kp = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2] + j * a.k_stride[1] + 8 * h;
                const T* vp = (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2] + j * a.v_stride[1] + 8 * h;
                const T* qp = (const T*)a.q + b * a.q_stride[0] + q.token * a.q_stride[1] + q.head * a.q_stride[2] + 8 * h;
                const T* gp = (const T*)a.dout + b * a.dout_stride[0] + q.token * a.dout_stride[1] + q.head * a.dout_stride[2] + 8 * h;
                acc16 z = acc16{}, dp = acc16{};
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    z = mma(load_frag(kp + 16 * s), load_frag(qp + 16 * s), z);
                    dp = mma(load_frag(vp + 16 * s), load_frag(gp + 16 * s), dp);
                }
                if (sp.cap2 > 0.f) cap_scores<16>(sp, z);
                else z *= sp.mul;
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = first + acc_row(r, lane);
                    float x = z[r] - lse2;
                    if (a.slopes) {
                        const float ak = a.at_k[b * a.at_k_stride[0] + hk * a.at_k_stride[1] + min(key, (int)a.keys - 1)];
                        x = fmaf(-(a.slopes[q.head] * kLog2e), fabsf(a.at_q[b * a.at_q_stride + q.token] - ak), x);
                    }
                    // (a key that the row does not see may hold anything)
                    sum += key >= lo && key <= hi ? weight2(x) * dp[r] : 0.f;
                }
                sum = half_sum(sum);
                if (left && hi < first + 32) {
                    delta = sum;
                    left = false;
                }
            }
            if (few && h == 0) out[RowPack::kDelta + i] = delta;
        }
    }
    if (h == 0) {
        out[RowPack::kLse + i] = lse2 < INFINITY ? fmaf(lse[stat], kLog2e, -shift) : INFINITY;
        out[RowPack::kLo + i] = __int_as_float(lo);
        out[RowPack::kHi + i] = __int_as_float(hi);
        out[RowPack::kSlope + i] = a.slopes ? a.slopes[q.head] * kLog2e : 0.f;
        out[RowPack::kAt + i] = a.slopes ? a.at_q[b * a.at_q_stride + q.token] : 0.f;
    }
    if (hk == 0) {
        const int first = col_min(some ? lo : INT_MAX), last = col_max(some ? hi : -1);
        const int flo = col_max(some ? lo : INT_MAX), fhi = col_min(some ? hi : -1);
        if (lane == 0) pack.bounds[b * pack.tiles + tile] = make_int4(first, last, flo, fhi);
    }
}

// The tiles of 32 query rows that see one of the keys first..last, in order,
// every parts-th from the part-th on; 64 bounds are looked at together, and
// the next 64 are on their way.  Every wavefront of a workgroup finds the same
// ones.
struct TileWalk {
    const int4* bounds;
    int tiles, first, last, base = -64, lane, parts, skip;
    int4 now, coming;
    uint64_t left = 0;
    __device__ inline TileWalk(const int4* b, int n, int first_, int last_, int part, int parts_, int lane_)
        : bounds(b), tiles(n), first(first_), last(last_), lane(lane_), parts(parts_), skip(part) {
        coming = bounds[min(lane, tiles - 1)];
    }
    // the next tile and its bounds, -1 after the last
    __device__ inline int next(int4* bd) {
        for (;;) {
            while (!left) {
                base += 64;
                if (base >= tiles) return -1;
                now = coming;
                if (base + 64 < tiles) coming = bounds[min(base + 64 + lane, tiles - 1)];
                left = __ballot(base + lane < tiles && now.x <= last && now.y >= first);
            }
            const int t = __builtin_ctzll(left);
            left &= left - 1;
            if (skip) {
                --skip;
                continue;
            }
            skip = parts - 1;
            *bd = make_int4(__builtin_amdgcn_readlane(now.x, t), __builtin_amdgcn_readlane(now.y, t), __builtin_amdgcn_readlane(now.z, t),
                            __builtin_amdgcn_readlane(now.w, t));
            return base + t;
        }
    }
};

// Sums of tiles of keys cut into parts of the query rows (parts 1: the pass
// writes its results itself): part s of key i of tile y (of all sequences), kv
// head h at index z = ((y * parts + s) * kv_heads + h) * kTileRows + i, D floats
// for dk at o[2 z D], as many for dv behind them; key weights: one float at o[z].
struct KeyParts {
    float* o;
    int parts;
    __device__ inline int64_t at(int64_t tile, int s, int kv_heads, int hk, int i) const { return ((tile * parts + s) * kv_heads + hk) * kTileRows + i; }
};

// f = 4 r (1 - r), r = 1 / (1 + exp2(c1 dot)): the derivative of the cap, of 16
// products z, which become the capped scores (kCapped: r, as in cap_shares)
template <Scores S>
__device__ inline void cap_slopes(const ScoreParams& sp, acc16& z, acc16& f) {
    auto each = [&](auto fine) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float y = z[i] * sp.mul, r = rcp_fast(1.f + exp2_fast(y)), r4 = 4.f * r;
            if constexpr (decltype(fine)::value) z[i] = fine_tanh(sp, y, r);
            else z[i] = S == kCapped ? r : fmaf(-2.f * sp.cap2, r, sp.cap2);
            f[i] = fmaf(-r4, r, r4);
        }
    };
    if (S == kAny && sp.fine) each(std::true_type{});
    else each(std::false_type{});
}

// One workgroup of W wavefronts, 32 keys each (a lane owns a key), over the
// tiles of 32 query rows that see them, all heads of the group: the sums over
// the group need no further pass, and no addition's order is left to chance.
// Query and dout rows are double buffered in LDS, keys stay in registers, values
// in LDS: with them there, addresses computed anew (fresh) and one product's
// registers given up before the next, two wavefronts a SIMD of 16-bit rows run
// without spilling (d = 128: 242 to 256 registers), one's products beside the
// other's exponentials.  Documents of 546 to 2,730 tokens, 16 heads, capped: 320
// us with one, 285 with two (with 1.5 of them on average, vector instructions
// active 43 % of the time, products 18 %); every key of 8,192 seen, no cap: a step
// 2.79 -> 2.66 ms, 750 to 825 TFLOP/s here (fp32, 4,096 tokens: 100).
//   Of 16-bit rows p and dx = p (dp - delta) are rounded to the type as factors of
// the second products, as in attend_tile (dx in two factors here and in attend_dq:
// 8,192 causal tokens, d = 64, 678 -> 785 us); an fp16 dx above 65,504 is infinite.
//   GRAD: dk = sum dx q, dv = sum p dout.  Else: w_out = w_in + sum p.
template <typename T, int D, Scores KIND, bool GRAD, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1)))
void attend_keys(frog_attend_t a, ScoreParams sp, int group, int key_tiles, RowPack pack, KeyParts parts, const int* order) {
    constexpr bool PLAIN = KIND == kPlain;
    constexpr int K = D / 16, M = D / 32;
    using L = Tile<T, D>;
    __shared__ __attribute__((aligned(16))) T q0[32 * D], q1[32 * D];
    __shared__ __attribute__((aligned(16))) T g0[GRAD ? 32 * D : 8], g1[GRAD ? 32 * D : 8];
    __shared__ __attribute__((aligned(16))) float p0[RowPack::kFloats], p1[RowPack::kFloats];
    __shared__ __attribute__((aligned(16))) T vl[GRAD ? 32 * W * D : 8];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int hk = (int)(blockIdx.x % (uint32_t)a.kv_heads), rows = (int)(a.queries * group);
    const uint32_t rest = blockIdx.x / (uint32_t)a.kv_heads;
    const Work work(order, rest, a.batch, key_tiles, parts.parts);
    // (without an order: earlier keys, which more queries see, first)
    const int tile = order ? work.tile : key_tiles - 1 - work.tile, part = work.part;
    const int64_t b = work.b, x = b * a.kv_heads + hk;
    const int first = tile * 32 * W, last = (int)min((int64_t)first + 32 * W, a.keys) - 1;
    const int j = first + w * 32 + (lane & 31), jc = min(j, last);
    const int wfirst = first + w * 32, wlast = wfirst + 31;
    frag<T> kf[K];
    {
        const T* p = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2] + jc * a.k_stride[1] + 8 * h;
#pragma unroll
        for (int s = 0; s < K; ++s) kf[s] = load_frag(p + 16 * s);
        if constexpr (GRAD)
            L::template load_rows<32 * W, W>(vl, w, lane, [&](int i) {
                return (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2] + min(first + i, last) * a.v_stride[1];
            });
    }
    const float ak = biased<KIND>(a.slopes) ? a.at_k[b * a.at_k_stride[0] + hk * a.at_k_stride[1] + jc] : 0.f;
    acc16 dk[GRAD ? M : 1], dv[GRAD ? M : 1];
    float sum = 0.f;
    if constexpr (GRAD) {
#pragma unroll
        for (int m = 0; m < M; ++m) dk[m] = dv[m] = acc16{};
    }
    const float* blocks = pack.rows + (int64_t)x * pack.tiles * RowPack::kFloats;
    TileWalk walk(pack.bounds + b * pack.tiles, pack.tiles, first, last, part, parts.parts, lane);

    // returns whether every row of the tile sees some key (else rows of zeros
    // stand in)
    auto fetch = [&](T* qs, T* gs, float* ps, int t, const int4& bd) {
        const T* zeros = (const T*)pack.zeros;
        const bool gaps = bd.z > bd.w;
        const float* blk = blocks + (int64_t)t * RowPack::kFloats;
        auto row = [&](const void* p, const int64_t(&st)[3], int i) {
            const QueryRow q(min(t * 32 + i, rows - 1), group, hk);
            const T* r = (const T*)p + b * st[0] + q.token * st[1] + q.head * st[2];
            if (gaps) r = blk[RowPack::kLse + i] < INFINITY ? r : zeros;
            return r;
        };
        L::template load_rows<32, W>(qs, w, lane, [&](int i) { return row(a.q, a.q_stride, i); });
        if constexpr (GRAD) L::template load_rows<32, W>(gs, w, lane, [&](int i) { return row(a.dout, a.dout_stride, i); });
        if (w == 0 && lane < RowPack::kFloats / 4)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(blk + 4 * lane), (__attribute__((address_space(3))) void*)ps,
                                             16, 0, 0);
    };
    auto step = [&](const T* qs, const T* gs, const float* ps, const int4& bd) {
        if (bd.x > wlast || bd.y < wfirst) return;
        const int from = fresh(lane);
        acc16 z = acc16{};
#pragma unroll
        for (int s = 0; s < K; ++s) z = mma(L::rows(qs, 0, s, from), kf[s], z);
        acc16 f;
        if constexpr (!PLAIN) {
            if (capped<KIND>(sp)) {
                cap_slopes<KIND>(sp, z, f);
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (KIND == kAny) f[r] = 1.f;
                    z[r] *= sp.mul;
                }
            }
            if (biased<KIND>(a.slopes)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const vec<float, 4> sl = *(const vec<float, 4>*)(ps + RowPack::kSlope + 8 * i + 4 * h);
                    const vec<float, 4> aq = *(const vec<float, 4>*)(ps + RowPack::kAt + 8 * i + 4 * h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[4 * i + e] = fmaf(-sl[e], fabsf(aq[e] - ak), z[4 * i + e]);
                }
            }
        }
        const float mul = KIND == kCapped ? -2.f * sp.cap2 : sp.mul;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const vec<float, 4> lse = *(const vec<float, 4>*)(ps + RowPack::kLse + 8 * i + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * i + e] = weight2(PLAIN || KIND == kCapped ? fmaf(z[4 * i + e], mul, -lse[e]) : z[4 * i + e] - lse[e]);
        }
        const bool whole = bd.z <= wfirst && bd.w >= wlast;
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const vec<float, 4> lo = *(const vec<float, 4>*)(ps + RowPack::kLo + 8 * i + 4 * h);
                const vec<float, 4> hi = *(const vec<float, 4>*)(ps + RowPack::kHi + 8 * i + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[4 * i + e] = j >= __float_as_int(lo[e]) && j <= __float_as_int(hi[e]) ? z[4 * i + e] : 0.f;
            }
        }
        if constexpr (GRAD) {
            // (the barriers keep the registers of one product from those of the
            // next: two wavefronts a SIMD overlap instead)
            __builtin_amdgcn_sched_barrier(0);
            int at = fresh(lane);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const frag<T> pf = to_frag<T>(z, t);
#pragma unroll
                for (int m = 0; m < M; ++m) dv[m] = mma(L::cols(gs, 16 * t, m, at), pf, dv[m]);
            }
            if constexpr (KIND == kCapped || KIND == kAny) {
#pragma unroll
                for (int r = 0; r < 16; ++r) z[r] = z[r] == 0.f ? 0.f : z[r] * f[r];
            }
            __builtin_amdgcn_sched_barrier(0);
            acc16 dp = acc16{};
            at = fresh(lane);
#pragma unroll
            for (int s = 0; s < K; ++s) dp = mma(L::rows(gs, 0, s, at), L::rows(vl, 32 * w, s, at), dp);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const vec<float, 4> delta = *(const vec<float, 4>*)(ps + RowPack::kDelta + 8 * i + 4 * h);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * i + e] -= delta[e];
            }
            // (a key without a query may hold anything: 0 times it is not 0)
            if (!whole) {
#pragma unroll
                for (int r = 0; r < 16; ++r) dp[r] = z[r] == 0.f ? 0.f : dp[r];
            }
            z *= dp;
            __builtin_amdgcn_sched_barrier(0);
            at = fresh(lane);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const frag<T> xf = to_frag<T>(z, t);
#pragma unroll
                for (int m = 0; m < M; ++m) dk[m] = mma(L::cols(qs, 16 * t, m, at), xf, dk[m]);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += z[r];
        }
    };
    auto ready = [&] {
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
    };
    int4 bd, bn;
    int t = walk.next(&bd);
    if (t >= 0) {
        fetch(q0, g0, p0, t, bd);
        for (;;) {
            ready();
            t = walk.next(&bn);
            if (t >= 0) fetch(q1, g1, p1, t, bn);
            step(q0, g0, p0, bd);
            if (t < 0) break;
            ready();
            t = walk.next(&bd);
            if (t >= 0) fetch(q0, g0, p0, t, bd);
            step(q1, g1, p1, bn);
            if (t < 0) break;
        }
    }
    if constexpr (GRAD) {
        if (j > last) return;
        if (parts.parts > 1) {
            float* po = parts.o + parts.at(b * key_tiles + tile, part, a.kv_heads, hk, j - first) * 2 * D + 4 * h;
            constexpr int to_dv = D;
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *(vec<float, 4>*)(po + 32 * m + 8 * i) = vec<float, 4>{dk[m][4 * i], dk[m][4 * i + 1], dk[m][4 * i + 2], dk[m][4 * i + 3]};
                    *(vec<float, 4>*)(po + to_dv + 32 * m + 8 * i) = vec<float, 4>{dv[m][4 * i], dv[m][4 * i + 1], dv[m][4 * i + 2], dv[m][4 * i + 3]};
                }
            return;
        }
        T* pk = (T*)a.dk + b * a.dk_stride[0] + hk * a.dk_stride[2] + j * a.dk_stride[1];
        T* pv = (T*)a.dv + b * a.dv_stride[0] + hk * a.dv_stride[2] + j * a.dv_stride[1];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                vec<T, 4> y, z;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[e] = (T)(dk[m][4 * i + e] * sp.scale);
                    z[e] = (T)dv[m][4 * i + e];
                }
                *(vec<T, 4>*)(pk + 32 * m + 8 * i + 4 * h) = y;
                *(vec<T, 4>*)(pv + 32 * m + 8 * i + 4 * h) = z;
            }
    } else {
        sum = half_sum(sum);
        if (j > last || lane >= 32) return;
        const int64_t at = (int64_t)x * a.keys + j;
        if (parts.parts > 1) parts.o[parts.at(b * key_tiles + tile, part, a.kv_heads, hk, j - first)] = sum;
        else a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + sum;
    }
}

// The parts of dk and dv summed, four values a thread; of the key weights, one.
template <typename T, int D, bool GRAD>
__global__ __launch_bounds__(256) void keys_join(frog_attend_t a, ScoreParams sp, int tiles, KeyParts parts) {
    constexpr int EACH = GRAD ? D / 2 : 1;      // threads a key
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, key = t / EACH;
    const int c = (int)(t % EACH), i = (int)(key % kTileRows), hk = (int)(key / kTileRows % a.kv_heads);
    const int64_t item = key / kTileRows / a.kv_heads, b = item / tiles, j = item % tiles * kTileRows + i;
    if (b >= a.batch || j >= a.keys) return;
    const float* p = parts.o + parts.at(item, 0, a.kv_heads, hk, i) * (GRAD ? 2 * D : 1);
    const int64_t step = (int64_t)a.kv_heads * kTileRows * (GRAD ? 2 * D : 1);
    if constexpr (GRAD) {
        vec<float, 4> y{};
#pragma unroll 4
        for (int s = 0; s < parts.parts; ++s) y += *(const vec<float, 4>*)(p + s * step + 4 * c);
        const bool second = c >= D / 4;
        if (!second) y *= sp.scale;
        vec<T, 4> x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (T)y[e];
        T* out = second ? (T*)a.dv + b * a.dv_stride[0] + j * a.dv_stride[1] + hk * a.dv_stride[2]
                        : (T*)a.dk + b * a.dk_stride[0] + j * a.dk_stride[1] + hk * a.dk_stride[2];
        *(vec<T, 4>*)(out + 4 * (second ? c - D / 4 : c)) = x;
    } else {
        float y = 0.f;
#pragma unroll 4
        for (int s = 0; s < parts.parts; ++s) y += p[s * step];
        const int64_t at = (b * a.kv_heads + hk) * a.keys + j;
        a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + y;
    }
}

// dq: one workgroup of W wavefronts, 32 query rows each (a lane owns a query),
// over the keys of their intervals in tiles of N, double buffered.  Three
// products a score and the exponentials beside them: 1,020 to 1,050 TFLOP/s at
// 8,192 tokens, 16 heads, d = 128, every key seen (fp32, 4,096 tokens: 113).
// Addresses computed anew (fresh) in every step take 30 registers and all spills
// from it: capped documents of 546 to 2,730 tokens 212 -> 163 us, every key seen
// without a cap 3 % slower.  dx is rounded as in attend_keys.
template <typename T, int D, Scores KIND, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1)))
void attend_dq(frog_attend_t a, ScoreParams sp, int group, int tiles, RowPack pack, const int* order) {
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
    const int hk = (int)(blockIdx.x % (uint32_t)a.kv_heads);
    const Work work(order, blockIdx.x / (uint32_t)a.kv_heads, a.batch, tiles, 1);
    const int tile = work.tile;
    const int64_t b = work.b, x = b * a.kv_heads + hk;
    const int64_t rows = a.queries * group, row = ((int64_t)tile * W + w) * 32 + (lane & 31);
    const QueryRow q(min(row, rows - 1), group, hk);
    int lo, hi;
    interval(a, b, q.token, &lo, &hi);
    const bool some = row < rows && lo <= hi;
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
    const T* kp = (const T*)a.k + b * a.k_stride[0] + hk * a.k_stride[2];
    const T* vp = (const T*)a.v + b * a.v_stride[0] + hk * a.v_stride[2];
    const float* akp = nullptr;
    float slope = 0.f, aq = 0.f;
    if (biased<KIND>(a.slopes)) {
        akp = a.at_k + b * a.at_k_stride[0] + hk * a.at_k_stride[1];
        slope = a.slopes[q.head] * kLog2e;
        aq = a.at_q[b * a.at_q_stride + q.token];
    }
    frag<T> qf[K], gf[K];
    {
        const T* p = (const T*)a.q + b * a.q_stride[0] + q.token * a.q_stride[1] + q.head * a.q_stride[2] + (lane >> 5) * 8;
        const T* g = (const T*)a.dout + b * a.dout_stride[0] + q.token * a.dout_stride[1] + q.head * a.dout_stride[2] + (lane >> 5) * 8;
#pragma unroll
        for (int s = 0; s < K; ++s) {
            qf[s] = load_frag(p + 16 * s);
            gf[s] = load_frag(g + 16 * s);
        }
    }
    // (a wavefront past the last row reads the last tile's numbers)
    const float* blk = pack.rows + ((int64_t)x * pack.tiles + min(tile * W + w, pack.tiles - 1)) * RowPack::kFloats + (lane & 31);
    const float lse = some ? blk[RowPack::kLse] : INFINITY, delta = blk[RowPack::kDelta];
    acc16 dq[M];
#pragma unroll
    for (int m = 0; m < M; ++m) dq[m] = acc16{};

    auto fetch = [&](T* ks, T* vs, float* as, int j) {
        L::template load<N, W>(ks, kp, a.k_stride[1], j, last, w, lane);
        L::template load<N, W>(vs, vp, a.v_stride[1], j, last, w, lane);
        if (biased<KIND>(akp) && w == 0)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(akp + min(j + lane, last)),
                                             (__attribute__((address_space(3))) void*)as, 4, 0, 0);
    };
    auto step = [&](const T* ks, const T* vs, const float* as, int j0) {
        if (j0 > whi || j0 + N <= wlo) return;
#pragma unroll
        for (int n = 0; n < S; ++n) {
            const int j = j0 + 32 * n;
            if (j > whi || j + 32 <= wlo) continue;
            acc16 z[1] = {acc16{}};
            int at = fresh(lane);
#pragma unroll
            for (int s = 0; s < K; ++s) z[0] = mma(L::rows(ks, 32 * n, s, at), qf[s], z[0]);
            // p (times the cap's slope), before the other product needs registers
            acc16 f{};
            if constexpr (!PLAIN) {
                if (capped<KIND>(sp)) {
                    cap_slopes<KIND>(sp, z[0], f);
                } else {
                    z[0] *= sp.mul;
                }
                if (biased<KIND>(akp)) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const vec<float, 4> ak = *(const vec<float, 4>*)(as + 32 * n + 8 * i + 4 * (lane >> 5));
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[0][4 * i + e] = fmaf(-slope, fabsf(aq - ak[e]), z[0][4 * i + e]);
                    }
                }
            }
            // (all rows here are finite: what no interval meets was cleared)
            if (j < flo || j + 31 > fhi) mask_scores<1>(z, lo - j, hi - j, lane, KIND == kCapped ? INFINITY : -INFINITY);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                z[0][r] = weight2(PLAIN || KIND == kCapped ? fmaf(z[0][r], KIND == kCapped ? -2.f * sp.cap2 : sp.mul, -lse) : z[0][r] - lse);
            if (capped<KIND>(sp)) z[0] *= f;
            acc16 dp = acc16{} - delta;
#pragma unroll
            for (int s = 0; s < K; ++s) dp = mma(L::rows(vs, 32 * n, s, at), gf[s], dp);
            dp *= z[0];
            at = fresh(lane);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const frag<T> xf = to_frag<T>(dp, t);
#pragma unroll
                for (int m = 0; m < M; ++m) dq[m] = mma(L::cols(ks, 32 * n + 16 * t, m, at), xf, dq[m]);
            }
        }
    };
    auto ready = [&] {
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
    };
    auto turn = [&](T* ks, T* vs, float* as, T* kn, T* vn, float* an, int j) {
        ready();
        if (j + N <= last) fetch(kn, vn, an, j + N);
        if (gaps) {
            rows_of.template clear<N, D, W>(ks, j, w, lane);
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
    if (row >= rows) return;
    T* out = (T*)a.dq + b * a.dq_stride[0] + q.token * a.dq_stride[1] + q.head * a.dq_stride[2];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vec<T, 4> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = some ? (T)(dq[m][4 * i + e] * sp.scale) : (T)0.f;
            *(vec<T, 4>*)(out + 32 * m + 8 * i + 4 * (lane >> 5)) = y;
        }
}

}  // namespace frog

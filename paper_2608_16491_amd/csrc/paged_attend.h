// Attention of one token per request over a cache in 8-bit pages: the kernels
// (instantiated per query type by paged_attend_*.hip) and how a call is cut.
//
// With code k = c 2^e and its row's power apart, a score is (q . c) 2^e: codes of
// both kinds are exact in bf16 (int8 7 bits, e4m3 4), so the products run on the
// bf16 matrix cores, q in one factor (bf16), two (fp16: 8 + 8 bits hold its 11)
// or three (fp32), and the power multiplies the sum.  A value's power multiplies
// its weight instead, and p 2^e enters the second product in two factors (16-bit
// queries: a weight is off by 2^-16 of itself at most) or three.
#pragma once

#include "attend_tile.h"
#include "paged.h"

namespace frog {

constexpr int kTile = 16, kTileShift = 4;   // keys of a tile; a step of a wavefront takes two
constexpr int kMostTiles = 256;       // of a workgroup's part of the cache
constexpr float kNoneSeen = -FLT_MAX; // running maximum of a row that has seen no key

// How a call is cut: parts of `chunk` tiles a workgroup, in parts of at most `tiles` tiles a request;
// `blocks` workgroups share the query rows of a kv head
struct PagedPlan {
    int64_t tiles;
    int chunk, parts, blocks, wide, waves;   // wide: two column tiles of 16 query rows
};

// Partial results (o null: one part, which writes the outputs itself): part s of
// row b * heads + h at [s * rows + row], o unnormalised
struct PagedParts {
    float* o;
    float2* ml;
    int64_t rows;
};

// The tiles request b's token walks, [first, end), and the rows it sees, [lo, hi]:
// tiles of the request's own pages in order, or of the listed pages
struct Walk {
    int64_t first, end;
    int lo, hi, last;     // last: where the query stands
    __device__ inline Walk(const frog_attend_paged_t& a, int64_t b) {
        lo = 0;
        hi = last = (int)rows_of(a.lengths, b, a.pages_per_request, a.cache.page) - 1;
        if (a.lr) {
            lo = max(lo, a.lr[2 * b]);
            hi = min(hi, a.lr[2 * b + 1]);
        }
        first = a.chosen ? 0 : lo / kTile;
        end = lo > hi ? first : a.chosen ? a.num_chosen * (a.cache.page / kTile) : hi / kTile + 1;
    }
};

// two floats whose upper halves are bf16 already
__device__ inline uint32_t upper_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); }

// eight codes as a factor
template <bool INT8>
__device__ inline frag<bf16_t> factor_of(uint32_t x, uint32_t y) {
    vec<uint32_t, 4> r;
    if constexpr (INT8) {
        const vec<float, 4> a = values_of<true>(x), b = values_of<true>(y);
        r = vec<uint32_t, 4>{upper_halves(a[0], a[1]), upper_halves(a[2], a[3]), upper_halves(b[0], b[1]), upper_halves(b[2], b[3])};
    } else {
        r = vec<uint32_t, 4>{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false)),
                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true)),
                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.f, false)),
                             __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, 1.f, true))};
    }
    return __builtin_bit_cast(frag<bf16_t>, r);
}

// byte N of the words of two rows, as a pair
template <bool INT8, int N>
__device__ inline uint32_t pair_of(uint32_t a, uint32_t b) {
    if constexpr (INT8) {
        return upper_halves((float)(int8_t)(a >> (8 * N)), (float)(int8_t)(b >> (8 * N)));
    } else {
        const uint32_t x = __builtin_amdgcn_perm(b, a, N < 2 ? 0x05010400 : 0x07030602);
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, (N & 1) != 0));
    }
}

// x in F factors of bf16
template <int F>
__device__ inline void split_factors(const vec<float, 8>& x, frag<bf16_t> (&f)[F]) {
    vec<float, 8> rest = x;
#pragma unroll
    for (int i = 0; i < F; ++i) {
        f[i] = __builtin_convertvector(rest, frag<bf16_t>);
        if (i + 1 < F) rest -= __builtin_convertvector(f[i], vec<float, 8>);
    }
}

// Columns of the score tiles: with at most G = 2, 4 or 8 query rows, rows repeat
// along the 16 columns, and the 8 scores a lane has of one are shared out: lane
// G j + g takes the E = G / 2 of part j, whose weights the others get from it.
// x of part J, in all lanes of the row of 16 that have the same g
template <int G, int J>
__device__ inline uint32_t from_part(uint32_t x) { return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, (J * G) << 5 | 0x10 | (G - 1)); }

// the part's own E of eight values
template <int E>
__device__ inline vec<float, E> own_part(vec<float, 8> x, int part) {
    vec<float, E> y;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        y[e] = x[e];
#pragma unroll
        for (int j = 1; j < 8 / E; ++j) y[e] = part == j ? x[j * E + e] : y[e];
    }
    return y;
}

// What the weights' two factors cost in products: where at most eight rows repeat
// along the columns, the first stands in columns 0 .. 7 of one product and the
// second in 8 .. 15, and the halves are added at the end (1,001 keys, four rows, d = 128:
// half of the second product's 16 matrix instructions a step).
template <int E, int F>
constexpr bool kHalves = E < 8 && F == 2;
template <int E, int F>
constexpr int kChains = kHalves<E, F> ? 1 : F;
// (the same for the queries' factors in the first product, whose halves are added at once)

// x of column ^ 8
__device__ inline float other_half(float x) { return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), 0x128, 0xF, 0xF, true)); }

// the factors of all eight weights from the part's own
template <int E, int F>
__device__ inline void share_factors(const vec<float, E>& p, frag<bf16_t> (&f)[kChains<E, F>], int col) {
    if constexpr (E == 8) {
        split_factors<F>(p, f);
    } else {
        constexpr int G = 2 * E;
        vec<float, E> rest = p;
        vec<bf16_t, E> own[F];
#pragma unroll
        for (int i = 0; i < F; ++i) {
            own[i] = __builtin_convertvector(rest, vec<bf16_t, E>);
            if (i + 1 < F) rest -= __builtin_convertvector(own[i], vec<float, E>);
        }
        auto gather = [](const uint32_t (&x)[E], uint32_t (&w)[8]) {
            // value e of part j: weight E j + e
#pragma unroll
            for (int e = 0; e < E; ++e) {
                w[e] = from_part<G, 0>(x[e]);
                w[E + e] = from_part<G, 1>(x[e]);
                if constexpr (E <= 2) {
                    w[2 * E + e] = from_part<G, 2>(x[e]);
                    w[3 * E + e] = from_part<G, 3>(x[e]);
                }
                if constexpr (E == 1) {
                    w[4] = from_part<G, 4>(x[e]);
                    w[5] = from_part<G, 5>(x[e]);
                    w[6] = from_part<G, 6>(x[e]);
                    w[7] = from_part<G, 7>(x[e]);
                }
            }
        };
        uint32_t x[E], w[8];
        vec<uint32_t, 4> a;
        if constexpr (F == 2) {
            // both factors of a weight in one word; a column takes its half of it
            const uint32_t half = col < 8 ? 0x05040100 : 0x07060302;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = __builtin_bit_cast(uint32_t, vec<bf16_t, 2>{own[0][e], own[1][e]});
            gather(x, w);
#pragma unroll
            for (int n = 0; n < 4; ++n) a[n] = __builtin_amdgcn_perm(w[2 * n + 1], w[2 * n], half);
            f[0] = __builtin_bit_cast(frag<bf16_t>, a);
        } else {
#pragma unroll
            for (int i = 0; i < F; ++i) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bf16_t y = own[i][e];      // (a bit cast of an element takes the vector's first)
                    x[e] = __builtin_bit_cast(uint16_t, y);
                }
                gather(x, w);
#pragma unroll
                for (int n = 0; n < 4; ++n) a[n] = __builtin_amdgcn_perm(w[2 * n + 1], w[2 * n], 0x05040100);
                f[i] = __builtin_bit_cast(frag<bf16_t>, a);
            }
        }
    }
}

// What a lane holds of a step's rows, as loaded.  Keys: of row lane % 16 of each
// tile the pieces that its quarter of the wavefront multiplies.  Values: of rows
// 4 (lane / 16) .. + 3 the bytes whose channels are row lane % 16 of the second
// product's left factor; slots of the quarter's 8 rows stand in the order of the
// score registers, so that no lane exchanges a value and nothing goes through LDS.
template <int D>
struct Rows {
    static constexpr int kV = D >= 96 ? 2 : 1;   // words of a value row
    uint32_t k[2][D / 16], v[2][4][kV], ke[2], ve[2];

    // first of the eight channels of product s
    __device__ static inline int channel(int s, int quarter) {
        if constexpr (D % 64 == 0) return 64 * (s / 2) + 16 * quarter + 8 * (s % 2);
        else return 32 * s + 8 * quarter;
    }
    // (blocks: of 16 rows of one head)
    __device__ inline void load_keys(const frog_cache_t& c, const int (&block)[2], int lane) {
        const int col = lane & 15, quarter = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t row = (int64_t)max(block[t], 0) * kTile;
            const uint8_t* p = (const uint8_t*)c.k + row * D;
            if constexpr (D % 64 == 0) {
#pragma unroll
                for (int i = 0; i < D / 64; ++i) *(uint4*)&k[t][4 * i] = *(const uint4*)(p + (uint32_t)(col * D + 16 * quarter) + 64 * i);
            } else {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) *(uint2*)&k[t][2 * i] = *(const uint2*)(p + (uint32_t)(col * D + 8 * quarter) + 32 * i);
            }
            ke[t] = *(const uint32_t*)(c.k_exp + row + 4 * quarter);
        }
    }
    __device__ inline void load_values(const frog_cache_t& c, const int (&block)[2], int lane) {
        const int col = lane & 15, quarter = lane >> 4;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t row = (int64_t)max(block[t], 0) * kTile;
            const uint8_t* p = (const uint8_t*)c.v + row * D;
            ve[t] = *(const uint32_t*)(c.v_exp + row + 4 * quarter);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t at = (uint32_t)(4 * quarter * D) + e * D;
                if constexpr (D == 128) *(uint2*)v[t][e] = *(const uint2*)(p + at + 8 * col);
                else if constexpr (D == 32) v[t][e][0] = *(const uint16_t*)(p + at + 2 * col);
                else v[t][e][0] = *(const uint32_t*)(p + at + 4 * col);
                if constexpr (D == 96) v[t][e][1] = *(const uint16_t*)(p + at + 64 + 2 * col);
            }
        }
    }
};

// the channel that value m of row i of the second product stands for (two
// neighbouring ones from an even m on)
template <int D>
__device__ inline int out_channel(int i, int m) {
    if constexpr (D == 96) return m < 4 ? 4 * i + m : 64 + 2 * i + m - 4;
    else return D / 16 * i + m;
}

// One workgroup of W wavefronts a (request, kv head, part of its rows).  A step of
// a wavefront is two tiles: their scores (keys x queries), one pass of the running
// maximum and sum, the second product with the values as they were loaded.  Many
// long requests are bound by HBM (32 of up to 40,000 rows, 32 / 8 heads, d = 128: 1.36
// GB in 248 us, 5.5 TB/s; vector instructions 30 % of the CUs' busy time, products
// 8 %); few query rows over d = 64 with a cap by vector instructions (65 %), of
// which half turn int8 codes into bf16; a single short request by the chain of
// a step (about 1 us).
//   Every tile of a part is walked, those of list entries that are none, of pages
// past a length and of pages outside lr among them (masked, with block 0's rows): a
// list costs what it has room for (48 requests of 300 to 1,000 rows, 32 / 8 heads, d = 128:
// without a list 21 us, with their pages in lists of 16 pages of 64 rows 26, of 64 60).
//   W = 4 with at most 128 registers (d = 128, up to eight query rows), four
// wavefronts a SIMD: a step's loads need only be one step ahead.  (fp16 of d = 128 and
// up to four query rows spills 1 to 9 registers there: 32 requests to 8,000 rows, 32 / 8
// heads, 73 us with the join, bf16 65.5.)  Two steps ahead
// took 78 us for 77 (chosen pages) and 11.2 for 10.4 (1,001 rows); W = 8 and 16 for
// long requests 5 to 20 % more, W = 2 the same for twice the parts.
template <typename T, bool INT8, int D, bool PLAIN, int E, int NQ, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(NQ == 2 || sizeof(T) == 4 ? 2 : W == 8 ? 2 : E < 8 ? 4 : 3)))
void paged_attend(frog_attend_paged_t a, ScoreParams sp, PagedPlan plan, PagedParts parts, uint32_t first_item) {
    constexpr int QF = sizeof(T) == 4 ? 3 : std::is_same<T, bf16_t>::value ? 1 : 2, PF = sizeof(T) == 4 ? 3 : 2;
    constexpr int M = D / 16, S = D / 32, G = 2 * E;
    static_assert(E == 8 || NQ == 1, "shared scores are of one column tile");
    __shared__ int block_of[kMostTiles], place_of[kMostTiles];
    __shared__ float tops[W][16 * NQ], sums[W][16 * NQ], most[16 * NQ], total[16 * NQ];
    // (rows apart by eight banks)
    constexpr int kRows = E < 8 ? G : 16 * NQ, kApart = D + 8;
    __shared__ __attribute__((aligned(16))) float joined[W][kRows * kApart];
    const frog_cache_t& c = a.cache;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quarter = lane >> 4, own = col / G;
    uint32_t item = first_item + blockIdx.x;
    const int h = (int)(item % (uint32_t)c.kv_heads);
    item /= (uint32_t)c.kv_heads;
    int rows0 = 0;
    if (plan.blocks > 1) {
        rows0 = (int)(item % (uint32_t)plan.blocks) * 16 * NQ;
        item /= (uint32_t)plan.blocks;
    }
    const int part = (int)(item % (uint32_t)plan.parts);
    const int64_t b = item / (uint32_t)plan.parts;
    const Walk walk(a, b);
    const int64_t first = walk.first + (int64_t)part * plan.chunk;
    const int count = (int)max((int64_t)0, min((int64_t)plan.chunk, walk.end - first));
    if (count == 0 && parts.o) return;
    const int group = a.heads / c.kv_heads, shift = shift_of(c.page) - kTileShift;      // a page's tiles: 1 << shift
    for (int i = threadIdx.x; i < ((count + 1) & ~1); i += 64 * W) {
        int block = -1, place = 0;
        if (i < count) {
            const int64_t entry = (first + i) >> shift;
            const int sub = (int)(first + i) & ((1 << shift) - 1);
            const int64_t logical = a.chosen ? a.chosen[(b * c.kv_heads + h) * a.num_chosen + entry] : entry;
            if (logical >= 0 && logical < a.pages_per_request) {
                place = (int)logical * c.page + sub * kTile;
                if (place <= walk.hi && place + kTile > walk.lo) {
                    const int page = page_of(a.pages, b, a.pages_per_request, logical, c.num_pages);
                    if (page >= 0) block = ((page * c.kv_heads + h) << shift) + sub;
                }
            }
        }
        block_of[i] = block;
        place_of[i] = place;
    }
    frag<bf16_t> qf[NQ][S][kChains<E, QF>];
    float slope[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int head = h * group + min(rows0 + 16 * n + col % G, group - 1);
        const T* p = (const T*)a.q + b * a.q_stride[0] + head * a.q_stride[1];
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const frag<T> x = load_frag(p + Rows<D>::channel(s, quarter));
            if constexpr (QF == 1) {
                qf[n][s][0] = x;
            } else if constexpr (kHalves<E, QF>) {
                frag<bf16_t> both[QF];
                split_factors<QF>(__builtin_convertvector(x, vec<float, 8>), both);
                qf[n][s][0] = col < 8 ? both[0] : both[1];
            } else {
                split_factors<QF>(__builtin_convertvector(x, vec<float, 8>), qf[n][s]);
            }
        }
        slope[n] = !PLAIN && a.slopes ? a.slopes[head] * kLog2e : 0.f;
    }
    acc4 o[NQ][M];
    float top[NQ], sum[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        top[n] = kNoneSeen;
        sum[n] = 0.f;
#pragma unroll
        for (int m = 0; m < M; ++m) o[n][m] = acc4{};
    }
    __syncthreads();

    struct Step {
        int block[2], place[2];
    };
    auto look = [&](int i) {
        Step s;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s.block[t] = __builtin_amdgcn_readfirstlane(block_of[i + t]);
            s.place[t] = __builtin_amdgcn_readfirstlane(place_of[i + t]);
        }
        return s;
    };
    auto step = [&](Rows<D>& r, const Step& at, const Step& next, bool more) __attribute__((always_inline)) {
        vec<float, 8> x[NQ];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            acc4 y[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n) y[n] = acc4{};
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const frag<bf16_t> k = factor_of<INT8>(r.k[t][2 * s], r.k[t][2 * s + 1]);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int f = 0; f < kChains<E, QF>; ++f) y[n] = mma(k, qf[n][s][f], y[n]);
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][4 * t + e] = kHalves<E, QF> ? y[n][e] + other_half(y[n][e]) : y[n][e];
        }
        // of the own scores: the powers' bytes, and where their keys stand
        const uint32_t ke0 = r.ke[0], ke1 = r.ke[1];
        if (more) r.load_keys(c, next.block, lane);
        auto byte_of = [&](uint32_t exps0, uint32_t exps1, int e) {
            if constexpr (E == 8) return ((e / 4 ? exps1 : exps0) >> (8 * (e % 4))) & 255;
            else return ((E * own >= 4 ? exps1 : exps0) >> (8 * ((E * own & 3) + e))) & 255;
        };
        auto tile_of = [&](int e) { return E == 8 ? e / 4 : E * own / 4; };
        auto place_of_key = [&](int e) {
            return (tile_of(e) ? at.place[1] : at.place[0]) + 4 * quarter + (E == 8 ? e % 4 : (E * own & 3) + e);
        };
        vec<float, E> z[NQ], up;
#pragma unroll
        for (int e = 0; e < E; ++e) up[e] = power_of(byte_of(r.ve[0], r.ve[1], e));
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            z[n] = own_part<E>(x[n], own);
#pragma unroll
            for (int e = 0; e < E; ++e) z[n][e] *= power_of(byte_of(ke0, ke1, e)) * (PLAIN ? sp.mul : 1.f);
            if constexpr (!PLAIN) {
                if (sp.cap2 > 0.f) cap_scores<E>(sp, z[n]);
                else z[n] *= sp.mul;
                if (a.slopes) {
#pragma unroll
                    for (int e = 0; e < E; ++e) z[n][e] -= slope[n] * fabsf((float)(walk.last - place_of_key(e)));
                }
            }
        }
        // rows outside lo .. hi, and of tiles that are none, may hold anything
        bool whole = true;
#pragma unroll
        for (int t = 0; t < 2; ++t) whole &= at.block[t] >= 0 && at.place[t] >= walk.lo && at.place[t] + kTile - 1 <= walk.hi;
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int place = at.place[e / 4] + 4 * quarter + e % 4;
                const bool seen = at.block[e / 4] >= 0 && place >= walk.lo && place <= walk.hi;
#pragma unroll
                for (int i = 0; i < Rows<D>::kV; ++i) r.v[e / 4][e % 4][i] = seen ? r.v[e / 4][e % 4][i] : 0;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int place = place_of_key(e);
                const bool seen = (tile_of(e) ? at.block[1] : at.block[0]) >= 0 && place >= walk.lo && place <= walk.hi;
                up[e] = seen ? up[e] : 0.f;
#pragma unroll
                for (int n = 0; n < NQ; ++n) z[n][e] = seen ? z[n][e] : -INFINITY;
            }
        }
        frag<bf16_t> pf[NQ][kChains<E, PF>];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float most = z[n][0];
#pragma unroll
            for (int e = 1; e < E; ++e) most = fmaxf(most, z[n][e]);
            // the maximum is renewed where it grew by more than 2^8
            if (__any(most > top[n] + 8.f)) {
                float now = fmaxf(most, top[n]);
#pragma unroll
                for (int i = G; i < 16; i *= 2) now = fmaxf(now, __shfl_xor(now, i));
                now = quarter_max(now);
                const float down = exp2_fast(top[n] - now);
                top[n] = now;
                sum[n] *= down;
#pragma unroll
                for (int m = 0; m < M; ++m) o[n][m] *= down;
            }
            vec<float, E> p;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                p[e] = exp2_fast(z[n][e] - top[n]);
                sum[n] += p[e];
            }
            share_factors<E, PF>(p * up, pf[n], col);
        }
        auto product = [&](auto byte, int word, int m) __attribute__((always_inline)) {
            constexpr int B = decltype(byte)::value;
            const vec<uint32_t, 4> x{pair_of<INT8, B>(r.v[0][0][word], r.v[0][1][word]), pair_of<INT8, B>(r.v[0][2][word], r.v[0][3][word]),
                                     pair_of<INT8, B>(r.v[1][0][word], r.v[1][1][word]), pair_of<INT8, B>(r.v[1][2][word], r.v[1][3][word])};
            const frag<bf16_t> v = __builtin_bit_cast(frag<bf16_t>, x);
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int f = 0; f < kChains<E, PF>; ++f) o[n][m] = mma(v, pf[n][f], o[n][m]);
        };
#pragma unroll
        for (int m = 0; m < M; m += 4) {
            product(std::integral_constant<int, 0>(), m / 4, m);
            product(std::integral_constant<int, 1>(), m / 4, m + 1);
            if (m + 2 < M) product(std::integral_constant<int, 2>(), m / 4, m + 2);
            if (m + 3 < M) product(std::integral_constant<int, 3>(), m / 4, m + 3);
        }
    };

    // a step's keys are loaded behind the scores of the one before, its values
    // behind the products of it (a tile that is none reads block 0: a cache has one)
    if (2 * w < count) {
        Rows<D> r;
        Step now = look(2 * w);
        r.load_keys(c, now.block, lane);
        r.load_values(c, now.block, lane);
        for (int i = 2 * w; i < count; i += 2 * W) {
            const bool more = i + 2 * W < count;
            const Step next = more ? look(i + 2 * W) : now;
            step(r, now, next, more);
            if (more) r.load_values(c, next.block, lane);
            now = next;
        }
    }

    // the wavefronts' results: maxima and sums, then every wavefront's outputs of
    // the rows there are, added by all threads
    const int rows = min(group - rows0, 16 * NQ);
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int i = G; i < 16; i *= 2) sum[n] += __shfl_xor(sum[n], i);
        sum[n] = quarter_sum(sum[n]);
        if (quarter == 0) {
            tops[w][16 * n + col] = top[n];
            sums[w][16 * n + col] = sum[n];
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        float all = kNoneSeen, sum_all = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) all = fmaxf(all, tops[i][16 * n + col]);
        if (w == 0) {
#pragma unroll
            for (int i = 0; i < W; ++i) sum_all += sums[i][16 * n + col] * exp2_fast(tops[i][16 * n + col] - all);
            if (quarter == 0) {
                most[16 * n + col] = all;
                total[16 * n + col] = sum_all;
            }
        }
        const float down = exp2_fast(top[n] - all);
        if constexpr (kHalves<E, PF>) {
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][m][e] += other_half(o[n][m][e]);
        }
        if (16 * n + col < rows) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int m = 0; m < M; m += 2)
                    *(float2*)&joined[w][(16 * n + col) * kApart + out_channel<D>(4 * quarter + e, m)] = make_float2(o[n][m][e] * down, o[n][m + 1][e] * down);
        }
    }
    __syncthreads();
    const int64_t row0 = b * a.heads + h * group + rows0;
    for (int i = threadIdx.x; i < rows * (D / 2); i += 64 * W) {
        const int row = i / (D / 2), channel = 2 * (i % (D / 2));
        float2 x = make_float2(0.f, 0.f);
#pragma unroll
        for (int n = 0; n < W; ++n) {
            const float2 y = *(const float2*)&joined[n][row * kApart + channel];
            x.x += y.x;
            x.y += y.y;
        }
        if (parts.o) {
            *(float2*)(parts.o + (part * parts.rows + row0 + row) * D + channel) = x;
        } else {
            const float scale = total[row] == 0.f ? 0.f : 1.f / total[row];
            *(vec<T, 2>*)((T*)a.out + b * a.out_stride[0] + (h * group + rows0 + row) * a.out_stride[1] + channel) = vec<T, 2>{(T)(x.x * scale), (T)(x.y * scale)};
        }
    }
    if (threadIdx.x < rows) {
        const float all = most[threadIdx.x], sum_all = total[threadIdx.x];
        if (parts.o) parts.ml[part * parts.rows + row0 + threadIdx.x] = make_float2(all, sum_all);
        else if (a.lse) a.lse[row0 + threadIdx.x] = sum_all == 0.f ? -INFINITY : (all + log2f(sum_all)) * kLn2;
    }
}

// launchers of one query type
hipError_t launch_paged_bf16(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream);
hipError_t launch_paged_f16(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream);
hipError_t launch_paged_f32(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream);

template <typename T, bool INT8, int D>
hipError_t launch_paged(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream) {
    const ScoreParams sp = score_params(a.scale, a.cap, a.type);
    const int64_t items = a.batch * plan.parts * plan.blocks * a.cache.kv_heads;
    auto run = [&](auto kernel, int threads) {
        return in_launches(items, threads, [&](int64_t first, dim3 grid) { kernel<<<grid, threads, 0, stream>>>(a, sp, plan, parts, (uint32_t)first); });
    };
    const bool plain = a.cap == 0.f && !a.slopes;
    if constexpr (sizeof(T) == 2) {
        if (plan.wide) return plain ? run(paged_attend<T, INT8, D, true, 8, 2, 4>, 256) : run(paged_attend<T, INT8, D, false, 8, 2, 4>, 256);
    }
    auto shared = [&](auto each) {
        constexpr int E = decltype(each)::value;
        if (plan.waves == 8) return plain ? run(paged_attend<T, INT8, D, true, E, 1, 8>, 512) : run(paged_attend<T, INT8, D, false, E, 1, 8>, 512);
        return plain ? run(paged_attend<T, INT8, D, true, E, 1, 4>, 256) : run(paged_attend<T, INT8, D, false, E, 1, 4>, 256);
    };
    const int group = a.heads / a.cache.kv_heads;
    if (group <= 2) return shared(std::integral_constant<int, 1>());
    if (group <= 4) return shared(std::integral_constant<int, 2>());
    if (group <= 8) return shared(std::integral_constant<int, 4>());
    return shared(std::integral_constant<int, 8>());
}

template <typename T>
hipError_t launch_paged_type(const frog_attend_paged_t& a, const PagedPlan& plan, const PagedParts& parts, hipStream_t stream) {
    auto codes = [&](auto d) {
        return a.cache.storage == FROG_CACHE_INT8 ? launch_paged<T, true, decltype(d)::value>(a, plan, parts, stream)
                                                  : launch_paged<T, false, decltype(d)::value>(a, plan, parts, stream);
    };
    switch (a.cache.d) {
        case 32: return codes(std::integral_constant<int, 32>());
        case 64: return codes(std::integral_constant<int, 64>());
        case 96: return codes(std::integral_constant<int, 96>());
        default: return codes(std::integral_constant<int, 128>());
    }
}

}  // namespace frog

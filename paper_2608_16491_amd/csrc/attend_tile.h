// Building blocks of the attention kernels on the matrix cores: fragments of
// 32 x 32 x 16 products for the three row types, LDS tiles of rows with their
// two ways of reading (by rows, and transposed), and the loads that fill them.
//
// Everywhere a lane owns one column of a product (a query in the forward pass
// and in dq, a key in dk and dv): in the accumulator of a 32 x 32 product lane
// L holds column L % 32 and, in register r, row 8 (r / 4) + 4 (L / 32) + r % 4.
// Softmax statistics are then per lane, and registers 8t .. 8t+7 of a score
// tile are, converted, the right factor of the next product over its rows
// 16t .. 16t+15, with slot e of half h standing for row 16t + 8 (e / 4) + 4 h
// + e % 4: the left factor is read with the same order, no lane exchanges a
// value.
#pragma once

#include <cfloat>
#include <climits>
#include <type_traits>

#include "attend.h"

namespace frog {

constexpr int kTileRows = 128;    // query rows (keys, in the passes that own keys) of a workgroup

using acc16 = vec<float, 16>;
template <typename T>
using frag = vec<T, 8>;

// c += a b over 16 values of the inner axis: half h of the wavefront holds
// slots 8h .. 8h+7 (in any order, the same for a and b)
__device__ inline acc16 mma(frag<bf16_t> a, frag<bf16_t> b, acc16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline acc16 mma(frag<f16_t> a, frag<f16_t> b, acc16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline acc16 mma(frag<float> a, frag<float> b, acc16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

template <typename T>
__device__ inline frag<T> to_frag(const acc16& c, int t) {
    vec<float, 8> x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = c[8 * t + e];
    if constexpr (sizeof(T) == 4) return x;
    else return __builtin_convertvector(x, frag<T>);
}

template <typename T>
__device__ inline frag<T> load_frag(const T* p) {   // 16-byte aligned
    if constexpr (sizeof(T) == 2) return *(const frag<T>*)p;
    else {
        const vec<float, 4> a = *(const vec<float, 4>*)p, b = *(const vec<float, 4>*)(p + 4);
        return frag<T>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
}

// C values from an address of their alignment (4, 8, 12, 16, 24 or 32 bytes).  A
// vector of six takes the memory of eight: what is copied is what was read.
template <typename T, int C>
__host__ __device__ inline vec<T, C> load_piece(const T* p) {
    constexpr int words = C * sizeof(T) / 4;
    uint32_t r[words];
    vec<T, C> x;
    static_assert(sizeof(r) == C * sizeof(T) && sizeof(r) <= sizeof(x), "whole words");
    if constexpr (words % 4 == 0) {
#pragma unroll
        for (int i = 0; i < words / 4; ++i) *(uint4*)(r + 4 * i) = ((const uint4*)p)[i];
    } else if constexpr (words % 2 == 0) {
#pragma unroll
        for (int i = 0; i < words / 2; ++i) *(uint2*)(r + 2 * i) = ((const uint2*)p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < words; ++i) r[i] = ((const uint32_t*)p)[i];
    }
    __builtin_memcpy(&x, r, sizeof(r));
    return x;
}

// what the rounding of x to the type leaves of it
template <typename T>
__device__ inline T rounded_off(float x) { return (T)(x - (float)(T)x); }

// N values of the output, and what their rounding left (frog_attend_t::out_low;
// none where `low` is null or rows are fp32)
template <typename T, int N, typename V>
__device__ inline void put_rounded(T* out, T* low, const V& x) {
    vec<T, N> y;
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = (T)x[e];
    *(vec<T, N>*)out = y;
    if constexpr (sizeof(T) == 2) {
        if (!low) return;
        vec<T, N> r;
#pragma unroll
        for (int e = 0; e < N; ++e) r[e] = rounded_off<T>(x[e]);
        *(vec<T, N>*)low = r;
    }
}

// max or sum over lanes L and L ^ 32, in both
__device__ inline float half_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float half_sum(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// over the 32 columns (lanes of one half; both halves hold the same)
__device__ inline int col_min(int x) {
    for (int o = 16; o; o >>= 1) x = min(x, __shfl_xor(x, o));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ inline int col_max(int x) {
    for (int o = 16; o; o >>= 1) x = max(x, __shfl_xor(x, o));
    return __builtin_amdgcn_readfirstlane(x);
}

// A tile of rows of D values in LDS, packed, the 16-byte pieces of a row
// permuted by an XOR with bits of the row's number so that the reads spread
// over all banks.
template <typename T, int D>
struct Tile {
    static constexpr int kPer = 16 / sizeof(T);   // values of a piece
    static constexpr int kPieces = D / kPer;      // pieces of a row: 4, 8, 12, 16, 24 or 32

    // Bits of the row's number for the XOR: 16 rows at one piece (row
    // fragments) and four rows at the four pieces of 64 bytes (the two reads
    // of 32 lanes of a transposed fragment) each cover 256 bytes of banks; of
    // 4-byte values rows r and r + 4 at eight pieces.  (With row % 16 alone a
    // transposed read of d = 128, bf16, took 10 cycles instead of 4, 60 % of
    // the cycles LDS was busy.)
    __device__ static inline int turn(int row) {
        if constexpr (kPieces % 16 == 0 && sizeof(T) == 4) return (row & 3) | ((row >> 1) & 4) | ((row << 1) & 8);
        else if constexpr (kPieces == 16) return ((row & 3) << 2) | ((row >> 2) & 3);
        else if constexpr (kPieces % 8 == 0 && sizeof(T) == 2) return ((row << 1) & 4) | ((row >> 2) & 3);
        else if constexpr (kPieces % 8 == 0) return (row >> 1) & 7;
        else return (row >> 2) & 3;
    }

    // rows [0, ROWS) of the tile from rows first + 0 .. of src (at most
    // `last`, which repeats), by direct loads into LDS; every wavefront w of W
    // takes its share.  Complete after a wait and a barrier.  A tile's rows
    // lie within 2 GiB (kMaxTokenStride): 32-bit offsets from its first.
    template <int ROWS, int W>
    __device__ static inline void load(T* lds, const T* src, int64_t stride, int first, int last, int w, int lane) {
        const char* base = (const char*)(src + (int64_t)first * stride);
        const uint32_t bytes = (uint32_t)stride * sizeof(T);
        const int most = last - first;
        constexpr int kLoads = ROWS * kPieces / 64;
#pragma unroll
        for (int i = 0; i < (kLoads + W - 1) / W; ++i) {
            const int c = i * W + w;
            if (kLoads % W && c >= kLoads) break;
            const int at = c * 64 + lane, row = at / kPieces, piece = at % kPieces;
            const uint32_t off = (uint32_t)min(row, most) * bytes + (piece ^ turn(row)) * 16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(base + off),
                                             (__attribute__((address_space(3))) void*)(lds + c * 64 * kPer), 16, 0, 0);
        }
    }

    // the same for scattered rows, with start(row) as the start of the tile's row
    template <int ROWS, int W, typename F>
    __device__ static inline void load_rows(T* lds, int w, int lane, F&& start) {
        constexpr int kLoads = ROWS * kPieces / 64;
        static_assert(ROWS * kPieces % 64 == 0, "whole wavefronts");
#pragma unroll
        for (int i = 0; i < (kLoads + W - 1) / W; ++i) {
            const int c = i * W + w;
            if (kLoads % W && c >= kLoads) break;
            const int at = c * 64 + lane, row = at / kPieces, piece = at % kPieces;
            const T* p = start(row) + (piece ^ turn(row)) * kPer;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                             (__attribute__((address_space(3))) void*)(lds + c * 64 * kPer), 16, 0, 0);
        }
    }

    // left factor by rows: rows base + lane % 32, values 16 s + 8 h ..
    __device__ static inline frag<T> rows(const T* lds, int base, int s, int lane) {
        const int row = base + (lane & 31), h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            return *(const frag<T>*)(lds + row * D + ((2 * s + h) ^ turn(row)) * kPer);
        } else {
            const vec<float, 4> a = *(const vec<float, 4>*)(lds + row * D + ((4 * s + 2 * h) ^ turn(row)) * kPer);
            const vec<float, 4> b = *(const vec<float, 4>*)(lds + row * D + ((4 * s + 2 * h + 1) ^ turn(row)) * kPer);
            return frag<T>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        }
    }

    // left factor transposed: value 32 m + lane % 32 of the 16 rows from base,
    // in the slot order of the accumulators
    __device__ static inline frag<T> cols(const T* lds, int base, int m, int lane) {
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // a transposing read hands 16 lanes four rows of 16 values
            using s4 = vec<short, 4>;
            const int i = lane & 15, piece = 4 * m + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
            vec<short, 8> out;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int row = base + 8 * q + 4 * h + (i >> 2);
                const T* p = lds + row * D + (piece ^ turn(row)) * kPer + (i & 1) * 4;
                const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)p);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[4 * q + e] = x[e];
            }
            return __builtin_bit_cast(frag<T>, out);
        } else {
            frag<T> out;
            const int c = 32 * m + (lane & 31);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = base + 8 * (e >> 2) + 4 * h + (e & 3);
                out[e] = lds[row * D + ((c / kPer) ^ turn(row)) * kPer + c % kPer];
            }
            return out;
        }
    }
};

// x, of which the compiler does not know that it is the same in every step of a
// loop: what is computed from it is not kept in registers between them
__device__ inline int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// row r of an accumulator register
__device__ inline int acc_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// Scores of keys outside lo..hi (numbers within the tile; the lane's query)
// become `out`.
template <int S>
__device__ inline void mask_scores(acc16 (&z)[S], int lo, int hi, int lane, float out) {
    const int at = 4 * (lane >> 5);
    lo -= at;
    hi -= at;
#pragma unroll
    for (int n = 0; n < S; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int c = 32 * n + acc_row(r, 0);
            z[n][r] = c >= lo && c <= hi ? z[n][r] : out;
        }
}

// The intervals of a workgroup's query rows, for tiles with keys that none of
// them sees between keys that some do: what such a row holds (anything) must
// not meet a weight of 0 in a product, so it becomes 0 in LDS.
template <int ROWS>
struct Gaps {
    int lo[ROWS], hi[ROWS];
    // whether there are any up to key `last`: a key after an interval's end
    // that no interval holds
    __device__ inline bool any(int last, int lane) const {
        bool gap = false;
        for (int i = lane; i < ROWS; i += 64) {
            const int j = hi[i] + 1;
            bool seen = lo[i] > hi[i] || j > last;
            for (int r = 0; r < ROWS; ++r) seen |= j >= lo[r] && j <= hi[r];
            gap |= !seen;
        }
        return __any(gap);
    }
    // rows j .. j + N - 1 of a tile of D values in LDS, by W wavefronts (call
    // between barriers)
    template <int N, int D, int W, typename T>
    __device__ inline void clear(T* tile, int j, int w, int lane) const {
        bool seen = false;
        for (int r = 0; r < ROWS; ++r) seen |= j + lane >= lo[r] && j + lane <= hi[r];
        const uint64_t all = __ballot(seen);
        for (int n = w; n < N; n += W) {
            if ((all >> n) & 1) continue;
            uint32_t* p = (uint32_t*)(tile + n * D);
            for (int c = lane; c < (int)(D * sizeof(T) / 4); c += 64) p[c] = 0;
        }
    }
};

// 16 x 16 x 32 products, for few query rows: lane L holds row / column L % 16
// and slots 8 (L / 16) .. + 7 of the inner axis of a factor; of the result
// column L % 16 and in register r row 4 (L / 16) + r.
using acc4 = vec<float, 4>;
__device__ inline acc4 mma(frag<bf16_t> a, frag<bf16_t> b, acc4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline acc4 mma(frag<f16_t> a, frag<f16_t> b, acc4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline acc4 mma(frag<float> a, frag<float> b, acc4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// over lanes L, L ^ 16, L ^ 32, L ^ 48, in all of them
__device__ inline float quarter_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ inline float quarter_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Query rows of one kv head: the group's heads of one token after another
// (row = token * group + head of the group), so that a tile's intervals are
// close together and keys are read once for all heads that share them.
struct QueryRow {
    int64_t token;
    int head;      // in 0 .. heads - 1
    __device__ inline QueryRow(int64_t row, int group, int kv_head) {
        token = (uint32_t)row / (uint32_t)group;
        head = kv_head * group + (int)((uint32_t)row % (uint32_t)group);
    }
};

// What a workgroup of a pass over tiles (of query rows or of keys) does: part
// `part` of tile `tile` of sequence b.  order (sequence * tiles + tile): longest
// first; null: later tiles first, which is that under a causal mask.
struct Work {
    int64_t b;
    int tile, part;
    __device__ inline Work(const int* order, uint32_t i, int64_t batch, int tiles, int parts) {
        part = (int)(i % (uint32_t)parts);
        const uint32_t rest = i / (uint32_t)parts;
        if (order) {
            const uint32_t item = (uint32_t)__builtin_amdgcn_readfirstlane(order[rest]);
            b = item / (uint32_t)tiles;
            tile = (int)(item % (uint32_t)tiles);
        } else {
            b = rest % (uint32_t)batch;
            tile = tiles - 1 - (int)(rest / (uint32_t)batch);
        }
    }
};

// the interval of a query clipped to the keys; empty: lo > hi
__device__ inline void interval(const frog_attend_t& a, int64_t b, int64_t token, int* lo, int* hi) {
    *lo = 0;
    *hi = (int)a.keys - 1;
    if (a.lr) {
        const int2 p = *(const int2*)(a.lr + b * a.lr_stride + 2 * token);
        *lo = max(*lo, p.x);
        *hi = min(*hi, p.y);
    }
}

}  // namespace frog

// A cache of keys and values in 8-bit pages (include/frog.h): views of the
// arguments and device helpers that the kernels writing, reading, choosing and
// attending over its pages share.
#pragma once

#include "attend.h"

namespace frog {

constexpr int kLeastExp = -100;       // of a row's power of two
constexpr int kNoRow = 255;           // the power's byte of a row that is not finite

// 2^(byte - 127); the byte 255 gives infinity, which the row's codes of 0 turn into NaN
__device__ inline float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// the power's byte of a row whose largest magnitude has these bits (m 2^n with
// 1 <= m < 2; the codes' limits are 1.75 2^8 and (1 + 63/64) 2^6)
template <bool INT8>
__device__ inline int power_byte(uint32_t bits) {
    constexpr int top = INT8 ? 6 : 8, part = INT8 ? 0x7E0000 : 0x600000;
    const int e = (int)(bits >> 23) - 127 - top + ((int)(bits & 0x7FFFFF) > part ? 1 : 0);
    return bits >= 0x7F800000u ? kNoRow : (e > kLeastExp ? e : kLeastExp) + 127;
}

// four codes of values within the limit, and their values
template <bool INT8>
__device__ inline uint32_t codes_of(float a, float b, float c, float d) {
    if constexpr (INT8) {
        // the sum's low byte is the integer nearest to the value, ties to even
        constexpr float magic = 12582912.f;     // 1.5 2^23
        const uint32_t x = __float_as_uint(a + magic), y = __float_as_uint(b + magic), z = __float_as_uint(c + magic), w = __float_as_uint(d + magic);
        const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x0C0C0400), hi = __builtin_amdgcn_perm(w, z, 0x04000C0C);
        return lo | hi;
    } else {
        int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    }
}

template <bool INT8>
__device__ inline vec<float, 4> values_of(uint32_t codes) {
    if constexpr (INT8) {
        return vec<float, 4>{(float)(int8_t)codes, (float)(int8_t)(codes >> 8), (float)(int8_t)(codes >> 16), (float)(int8_t)(codes >> 24)};
    } else {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
        return vec<float, 4>{a[0], a[1], b[0], b[1]};
    }
}

// How a row is spread over lanes by the kernels that walk whole rows: kLanes
// neighbouring lanes of kEach values (8 or 12), so that 16-bit values load in
// pieces of 16 or 24 bytes and codes in 8 or 12.
template <int D>
struct RowSplit {
    static constexpr int kEach = D == 96 ? 12 : 8, kLanes = D / kEach, kRows = 64 / kLanes;   // kRows: of one wavefront
};

// over the L lanes of a row (4, 8 or 16, aligned): by exchanges inside a row of 16 lanes
template <int L, typename F>
__device__ inline uint32_t over_row(uint32_t x, F&& f) {
    x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));                   // lanes ^ 1
    x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));                   // lanes ^ 2
    if constexpr (L >= 8) x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true));    // the other half of 8
    if constexpr (L >= 16) x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true));   // the other half of 16
    return x;
}

// N words at p, on a boundary of 16, 8 or 4 bytes as N divides; `streamed`: past the
// caches where they are not looked for again soon (writing prompts of 639 MB 134
// -> 131 us, reading 1.08 GB back 225 -> 210; rows that the attention after it
// finds in the caches are no longer there, which costs it about as much)
template <int N>
struct Words {
    uint32_t w[N];
};
template <int N, bool STREAMED = false>
__device__ inline Words<N> load_words(const void* p) {
    constexpr int M = N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    using V = vec<uint32_t, M>;
    Words<N> r;
#pragma unroll
    for (int i = 0; i < N / M; ++i) {
        const V x = STREAMED ? __builtin_nontemporal_load((const V*)p + i) : ((const V*)p)[i];
#pragma unroll
        for (int e = 0; e < M; ++e) r.w[M * i + e] = x[e];
    }
    return r;
}
template <int N>
__device__ inline void store_words(void* p, const Words<N>& r) {
    constexpr int M = N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    using V = vec<uint32_t, M>;
#pragma unroll
    for (int i = 0; i < N / M; ++i) {
        V x;
#pragma unroll
        for (int e = 0; e < M; ++e) x[e] = r.w[M * i + e];
        ((V*)p)[i] = x;
    }
}
template <int N>
__device__ inline void store_streamed(void* p, const Words<N>& r) {
    constexpr int M = N % 4 == 0 ? 4 : N % 2 == 0 ? 2 : 1;
    using V = vec<uint32_t, M>;
#pragma unroll
    for (int i = 0; i < N / M; ++i) {
        V x;
#pragma unroll
        for (int e = 0; e < M; ++e) x[e] = r.w[M * i + e];
        __builtin_nontemporal_store(x, (V*)p + i);
    }
}

// N values of a row as floats (16-bit ones: pieces of 16 or 8 bytes)
template <typename T, int N>
__device__ inline void load_values(const T* p, float (&x)[N]) {
    const Words<N * sizeof(T) / 4> r = load_words<N * sizeof(T) / 4, true>(p);
    T y[N];
    static_assert(sizeof(y) == sizeof(r), "whole words");
    __builtin_memcpy(y, r.w, sizeof(y));
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)y[i];
}

// pages are powers of two: row t stands in page t >> shift
__device__ inline int shift_of(int page) { return __builtin_ctz((unsigned)page); }

// rows of request b, clipped to its pages
__device__ inline int64_t rows_of(const int32_t* lengths, int64_t b, int64_t pages_per_request, int page) {
    return max((int64_t)0, min((int64_t)lengths[b], pages_per_request * page));
}

// page `at` of request b; -1: none
__device__ inline int page_of(const int32_t* pages, int64_t b, int64_t pages_per_request, int64_t at, int64_t num_pages) {
    const int p = pages[b * pages_per_request + at];
    return p >= 0 && p < num_pages ? p : -1;
}

// launchers: the arguments have been checked (paged_api.cpp), and the matching
// *_ws call, which gives the bytes of ws, has not refused the call's grids
int launch_cache_write(const frog_cache_write_t& a, hipStream_t stream);
int launch_cache_read(const frog_cache_read_t& a, hipStream_t stream);
int64_t select_pages_ws(const frog_select_pages_t& a);
int launch_select_pages(const frog_select_pages_t& a, void* ws, hipStream_t stream);
int64_t attend_paged_ws(const frog_attend_paged_t& a);
int launch_attend_paged(const frog_attend_paged_t& a, void* ws, hipStream_t stream);

}  // namespace frog

// What the C entry points of the attention and of the paged-cache sections of
// include/frog.h share: argument checks, the call's workspace, and the guard
// that lets nothing thrown leave the library.
#pragma once

#include <cmath>
#include <exception>
#include <new>

#include "attend.h"
#include "ws_pool.h"

namespace frog {

constexpr int64_t kMaxRows = (int64_t)1 << 30;  // keys, queries x group: 32-bit row numbers in the kernels
constexpr int64_t kMaxGrid = 0x7fffffff;

inline bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// row starts of a tensor of n[0..N) rows at strides s: 16-byte boundaries (the
// stride of an axis of one row is not used)
template <int N>
int check_rows(const char* name, const void* p, const int64_t (&s)[N], const int64_t (&n)[N], int size) {
    if (!p) return fail(FROG_EINVAL, "%s is NULL", name);
    if (misaligned(p)) return fail(FROG_EINVAL, "%s does not start on a 16-byte boundary", name);
    for (int i = 0; i < N; ++i)
        if (n[i] > 1 && (s[i] < 0 || (s[i] * size) % 16)) return fail(FROG_EINVAL, "%s: stride %lld is negative or not a multiple of 16 bytes", name, (long long)s[i]);
    return FROG_OK;
}

inline int check_type(int type, int* size) {
    if (type != FROG_STORAGE_F32 && type != FROG_STORAGE_F16 && type != FROG_STORAGE_BF16) return fail(FROG_EINVAL, "type %d: one of FROG_STORAGE_*", type);
    *size = type == FROG_STORAGE_F32 ? 4 : 2;
    return FROG_OK;
}

inline int check_heads(int heads, int kv_heads, int d, float scale, float cap) {
    if (heads < 1 || kv_heads < 1 || heads % kv_heads) return fail(FROG_EINVAL, "heads %d, kv_heads %d: the second must divide the first", heads, kv_heads);
    if (heads > 65535) return fail(FROG_EUNSUPPORTED, "heads %d > 65535", heads);
    if (d != 32 && d != 64 && d != 96 && d != 128) return fail(FROG_EUNSUPPORTED, "d %d: 32, 64, 96 or 128", d);
    if (!std::isfinite(scale)) return fail(FROG_EINVAL, "scale is not finite");
    if (!std::isfinite(cap) || cap < 0.f) return fail(FROG_EINVAL, "cap must be finite and >= 0");
    if (cap > 0.f && !(std::isfinite(4.f * scale / cap) && std::isfinite(4.f * cap))) return fail(FROG_EINVAL, "cap %g: scale / cap or cap overflows", (double)cap);
    return FROG_OK;
}

#define TRY(expr)                     \
    do {                              \
        int rc_ = (expr);             \
        if (rc_ != FROG_OK) return rc_; \
    } while (0)

// the call's workspace (the caller's, or the stream's buffer of the library)
// around its launches
template <typename A, typename F>
int with_ws(const A& a, int64_t bytes, hipStream_t stream, F&& launch) {
    if (bytes < 0) return (int)bytes;
    if (bytes == 0) return launch(nullptr);
    if (a.ws) {
        if ((uintptr_t)a.ws & 255) return fail(FROG_EINVAL, "the workspace does not start on a 256-byte boundary");
        if (a.ws_bytes < bytes) return fail(FROG_EINVAL, "workspace of %lld bytes, %lld needed", (long long)a.ws_bytes, (long long)bytes);
        return launch(a.ws);
    }
    // A graph outlives the call, and the library's buffer may be freed for a
    // larger one or serve another call between replays.
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    hipError_t e = hipStreamIsCapturing(stream, &capture);
    if (e != hipSuccess) return fail(FROG_EHIP, "capture status of the stream: %s", hipGetErrorString(e));
    if (capture != hipStreamCaptureStatusNone) return fail(FROG_EINVAL, "a call under graph capture takes the caller's workspace (%lld bytes)", (long long)bytes);
    WsLease lease;
    void* p = nullptr;
    e = lease.acquire(stream, (size_t)bytes, &p);
    if (e != hipSuccess) return fail(e == hipErrorOutOfMemory ? FROG_ENOMEM : FROG_EHIP, "workspace of %lld bytes: %s", (long long)bytes, hipGetErrorString(e));
    return launch(p);
}

// nothing thrown on the way (the workspace table allocates) leaves the library
template <typename F>
auto guarded(F&& f) -> decltype(f()) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(FROG_ENOMEM, "out of host memory");
    } catch (const std::exception& e) {
        return fail(FROG_EHIP, "%s", e.what());
    }
}

}  // namespace frog

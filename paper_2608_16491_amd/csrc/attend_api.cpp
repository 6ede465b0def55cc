// extern "C" entry points of the attention section of include/frog.h:
// argument checks, workspace, dispatch to the launchers.

#include <cmath>

#include "attend.h"
#include "ws_pool.h"

namespace frog {
namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30;  // keys, queries x group: 32-bit row numbers in the kernels
constexpr int64_t kMaxGrid = 0x7fffffff;

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

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

int check_type(int type, int* size) {
    if (type != FROG_STORAGE_F32 && type != FROG_STORAGE_F16 && type != FROG_STORAGE_BF16) return fail(FROG_EINVAL, "type %d: one of FROG_STORAGE_*", type);
    *size = type == FROG_STORAGE_F32 ? 4 : 2;
    return FROG_OK;
}

int check_heads(int heads, int kv_heads, int d, float scale, float cap) {
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

int check_attend(const frog_attend_t* a, bool backward) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    TRY(check_heads(a->heads, a->kv_heads, a->d, a->scale, a->cap));
    if (a->batch < 0 || a->queries < 0 || a->keys < 0) return fail(FROG_EINVAL, "negative size");
    const int64_t group = a->heads / a->kv_heads;
    if (a->keys > kMaxRows || a->queries > kMaxRows / group) return fail(FROG_EUNSUPPORTED, "more than 2^30 keys or query rows per kv head");
    if (a->batch > kMaxGrid / a->heads) return fail(FROG_EUNSUPPORTED, "batch * heads exceeds 2^31");
    if (a->batch == 0) return FROG_OK;
    const int64_t rows[3] = {a->batch, a->queries, a->heads}, cols[3] = {a->batch, a->keys, a->kv_heads};
    if (a->queries > 0) {
        TRY(check_rows("q", a->q, a->q_stride, rows, size));
        TRY(check_rows("out", a->out, a->out_stride, rows, size));
        if (a->out_low && size == 2) TRY(check_rows("out_low", a->out_low, a->out_stride, rows, size));
    }
    if (a->keys > 0) {
        TRY(check_rows("k", a->k, a->k_stride, cols, size));
        TRY(check_rows("v", a->v, a->v_stride, cols, size));
    }
    const int64_t far = kMaxTokenStride / size;
    if ((a->keys > 1 && (a->k_stride[1] > far || a->v_stride[1] > far))) return fail(FROG_EUNSUPPORTED, "k or v: rows more than 16 MiB apart");
    if (a->lr_stride < 0 || a->at_q_stride < 0 || a->at_k_stride[0] < 0 || a->at_k_stride[1] < 0) return fail(FROG_EINVAL, "negative stride");
    if (((uintptr_t)a->lr & 7) || (a->lr_stride & 1)) return fail(FROG_EINVAL, "lr: intervals must start on 8-byte boundaries");
    if (a->slopes && ((a->queries > 0 && !a->at_q) || (a->keys > 0 && !a->at_k))) return fail(FROG_EINVAL, "slopes need at_q and at_k");
    if (!a->slopes && (a->at_q || a->at_k)) return fail(FROG_EINVAL, "at_q and at_k need slopes");
    if (a->w_in && !a->w_out) return fail(FROG_EINVAL, "w_in needs w_out");
    if (backward) {
        if (a->w_in || a->w_out) return fail(FROG_EINVAL, "the backward pass takes no weights");
        if (a->queries > 0) {
            TRY(check_rows("dout", a->dout, a->dout_stride, rows, size));
            TRY(check_rows("dq", a->dq, a->dq_stride, rows, size));
            if (!a->lse) return fail(FROG_EINVAL, "lse is NULL");
        }
        if (a->keys > 0) {
            TRY(check_rows("dk", a->dk, a->dk_stride, cols, size));
            TRY(check_rows("dv", a->dv, a->dv_stride, cols, size));
        }
    }
    return FROG_OK;
}

int check_shared(const frog_attend_shared_t* a) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    TRY(check_heads(a->heads, a->kv_heads, a->d, a->scale, a->cap));
    if (a->batch < 0 || a->prefix < 0 || a->num_pages < 0 || a->pages_per_request < 0) return fail(FROG_EINVAL, "negative size");
    if (a->pages_per_request > 0 && a->page < 1) return fail(FROG_EINVAL, "page %d < 1", a->page);
    if (a->prefix > kMaxRows || a->batch > kMaxRows / a->heads || a->num_pages > 0x7fffffff) return fail(FROG_EUNSUPPORTED, "more than 2^30 prefix rows or query rows");
    if (a->pages_per_request > 0 && a->pages_per_request > kMaxRows / a->page) return fail(FROG_EUNSUPPORTED, "more than 2^30 tail rows");
    if (a->batch == 0) return FROG_OK;
    const int64_t rows[2] = {a->batch, a->heads}, cols[2] = {a->prefix, a->kv_heads}, paged[3] = {a->num_pages, a->page, a->kv_heads};
    TRY(check_rows("q", a->q, a->q_stride, rows, size));
    TRY(check_rows("out", a->out, a->out_stride, rows, size));
    if (a->prefix > 0) {
        TRY(check_rows("k", a->k, a->k_stride, cols, size));
        TRY(check_rows("v", a->v, a->v_stride, cols, size));
    }
    if (a->prefix > 1 && (a->k_stride[0] > kMaxTokenStride / size || a->v_stride[0] > kMaxTokenStride / size))
        return fail(FROG_EUNSUPPORTED, "k or v: rows more than 16 MiB apart");
    if (a->pages_per_request > 0) {
        if (!a->pages || !a->lengths) return fail(FROG_EINVAL, "pages or lengths is NULL");
        if (a->num_pages > 0) {
            TRY(check_rows("k_pages", a->k_pages, a->k_pages_stride, paged, size));
            TRY(check_rows("v_pages", a->v_pages, a->v_pages_stride, paged, size));
        }
    }
    if ((uintptr_t)a->lr & 7) return fail(FROG_EINVAL, "lr: intervals must start on 8-byte boundaries");
    return FROG_OK;
}

int check_evict(const frog_evict_t* a) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    if (a->batch < 0 || a->slots < 0 || a->heads < 1 || a->d < 1) return fail(FROG_EINVAL, "negative size");
    if ((int64_t)a->d * size % 16) return fail(FROG_EUNSUPPORTED, "d %d: rows must be a multiple of 16 bytes", a->d);
    if (a->recent < 0 || a->recent > a->keep || a->keep > a->slots) return fail(FROG_EINVAL, "0 <= recent <= keep <= slots is violated");
    if (a->slots > kMaxRows || a->heads > 65535 || a->batch > kMaxGrid / a->heads) return fail(FROG_EUNSUPPORTED, "more than 2^30 slots or 2^31 caches");
    if (a->batch == 0) return FROG_OK;
    if (!a->lengths || !a->lengths_out) return fail(FROG_EINVAL, "lengths or lengths_out is NULL");
    if (a->keep == 0) return FROG_OK;
    const int64_t cols[3] = {a->batch, a->slots, a->heads};
    TRY(check_rows("k", a->k, a->k_stride, cols, size));
    TRY(check_rows("v", a->v, a->v_stride, cols, size));
    if (!a->weights || !a->weights_out || !a->positions_out) return fail(FROG_EINVAL, "weights, weights_out or positions_out is NULL");
    if (!a->k_out || !a->v_out || misaligned(a->k_out) || misaligned(a->v_out)) return fail(FROG_EINVAL, "k_out or v_out is NULL or not on a 16-byte boundary");
    return FROG_OK;
}

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

}  // namespace
}  // namespace frog

using namespace frog;

extern "C" {

int64_t frog_attend_workspace(const frog_attend_t* a, int backward) {
    clear_error();
    int rc = check_attend(a, backward != 0);
    if (rc != FROG_OK) return rc;
    return backward ? attend_bwd_ws(*a) : attend_ws(*a);
}

int frog_attend(const frog_attend_t* a, void* stream) {
    clear_error();
    TRY(check_attend(a, false));
    return guarded([&] { return with_ws(*a, attend_ws(*a), (hipStream_t)stream, [&](void* ws) { return launch_attend(*a, ws, (hipStream_t)stream); }); });
}

int frog_attend_backward(const frog_attend_t* a, void* stream) {
    clear_error();
    TRY(check_attend(a, true));
    return guarded([&] { return with_ws(*a, attend_bwd_ws(*a), (hipStream_t)stream, [&](void* ws) { return launch_attend_bwd(*a, ws, (hipStream_t)stream); }); });
}

int64_t frog_attend_shared_workspace(const frog_attend_shared_t* a) {
    clear_error();
    int rc = check_shared(a);
    return rc != FROG_OK ? rc : attend_shared_ws(*a);
}

int frog_attend_shared(const frog_attend_shared_t* a, void* stream) {
    clear_error();
    TRY(check_shared(a));
    return guarded([&] { return with_ws(*a, attend_shared_ws(*a), (hipStream_t)stream, [&](void* ws) { return launch_attend_shared(*a, ws, (hipStream_t)stream); }); });
}

int64_t frog_evict_workspace(const frog_evict_t* a) {
    clear_error();
    int rc = check_evict(a);
    return rc != FROG_OK ? rc : evict_ws(*a);
}

int frog_evict(const frog_evict_t* a, void* stream) {
    clear_error();
    TRY(check_evict(a));
    return guarded([&] { return with_ws(*a, evict_ws(*a), (hipStream_t)stream, [&](void* ws) { return launch_evict(*a, ws, (hipStream_t)stream); }); });
}

}  // extern "C"

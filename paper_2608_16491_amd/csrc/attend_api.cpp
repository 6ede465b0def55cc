// extern "C" entry points of the attention section of include/frog.h:
// argument checks, workspace, dispatch to the launchers.

#include "api_checks.h"

namespace frog {
namespace {

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

// extern "C" entry points of the paged-cache section of include/frog.h:
// argument checks, workspace, dispatch to the launchers.

#include "api_checks.h"
#include "paged.h"

namespace frog {
namespace {

// `rows`, `bounds`: whether the call reads or writes them
int check_cache(const frog_cache_t& c, bool rows, bool bounds) {
    if (c.storage != FROG_CACHE_E4M3 && c.storage != FROG_CACHE_INT8) return fail(FROG_EINVAL, "storage %d: one of FROG_CACHE_*", c.storage);
    if (c.num_pages < 0 || c.kv_heads < 1) return fail(FROG_EINVAL, "a cache of %lld pages, %d kv heads", (long long)c.num_pages, c.kv_heads);
    if (c.page != 16 && c.page != 32 && c.page != 64 && c.page != 128 && c.page != 256) return fail(FROG_EINVAL, "page %d: 16, 32, 64, 128 or 256", c.page);
    if (c.d != 32 && c.d != 64 && c.d != 96 && c.d != 128) return fail(FROG_EUNSUPPORTED, "d %d: 32, 64, 96 or 128", c.d);
    if (c.kv_heads > 65535 || c.num_pages > kMaxGrid || c.num_pages * c.page >= ((int64_t)1 << 35) / c.kv_heads)
        return fail(FROG_EUNSUPPORTED, "a cache of 2^35 rows or more");
    if (c.num_pages == 0) return FROG_OK;
    if (rows) {
        if (!c.k || !c.v || !c.k_exp || !c.v_exp) return fail(FROG_EINVAL, "an array of the cache is NULL");
        if (misaligned(c.k) || misaligned(c.v) || misaligned(c.k_exp) || misaligned(c.v_exp)) return fail(FROG_EINVAL, "an array of the cache does not start on a 16-byte boundary");
    }
    if (bounds && !c.bounds) return fail(FROG_EINVAL, "the cache keeps no bounds");
    if (misaligned(c.bounds)) return fail(FROG_EINVAL, "the cache's bounds do not start on a 16-byte boundary");
    return FROG_OK;
}

template <typename A>
int check_requests(const A& a) {
    if (a.batch < 0 || a.pages_per_request < 0) return fail(FROG_EINVAL, "negative size");
    if (a.batch > kMaxRows || a.pages_per_request > kMaxRows / a.cache.page) return fail(FROG_EUNSUPPORTED, "more than 2^30 requests, or rows a request");
    if (a.batch == 0) return FROG_OK;
    if (!a.lengths || (a.pages_per_request > 0 && !a.pages)) return fail(FROG_EINVAL, "pages or lengths is NULL");
    return FROG_OK;
}

int check_queries(const void* q, const int64_t (&stride)[2], int64_t batch, int heads, const frog_cache_t& c, int size) {
    if (heads < 1 || heads % c.kv_heads) return fail(FROG_EINVAL, "heads %d, kv_heads %d: the second must divide the first", heads, c.kv_heads);
    if (heads > 65535) return fail(FROG_EUNSUPPORTED, "heads %d > 65535", heads);
    if (batch > kMaxGrid / heads) return fail(FROG_EUNSUPPORTED, "batch * heads exceeds 2^31");
    const int64_t rows[2] = {batch, heads};
    return batch ? check_rows("q", q, stride, rows, size) : FROG_OK;
}

int check_write(const frog_cache_write_t* a) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    TRY(check_cache(a->cache, true, false));
    TRY(check_requests(*a));
    if (a->tokens < 0) return fail(FROG_EINVAL, "negative size");
    if (a->tokens > 0x7fffffff) return fail(FROG_EUNSUPPORTED, "more than 2^31 rows");
    if (a->batch == 0 || a->tokens == 0) return FROG_OK;
    if (!a->starts && a->tokens % a->batch) return fail(FROG_EINVAL, "%lld rows are no equal shares of %lld requests", (long long)a->tokens, (long long)a->batch);
    const int64_t rows[2] = {a->tokens, a->cache.kv_heads};
    TRY(check_rows("k", a->k, a->k_stride, rows, size));
    return check_rows("v", a->v, a->v_stride, rows, size);
}

int check_read(const frog_cache_read_t* a) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    TRY(check_cache(a->cache, true, false));
    TRY(check_requests(*a));
    if (a->slots < 0) return fail(FROG_EINVAL, "negative size");
    if (a->slots > kMaxRows) return fail(FROG_EUNSUPPORTED, "more than 2^30 rows a request");
    if (a->batch == 0 || a->slots == 0) return FROG_OK;
    const int64_t rows[3] = {a->batch, a->slots, a->cache.kv_heads};
    TRY(check_rows("k", a->k, a->k_stride, rows, size));
    return check_rows("v", a->v, a->v_stride, rows, size);
}

int check_select(const frog_select_pages_t* a) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    TRY(check_cache(a->cache, false, true));
    TRY(check_requests(*a));
    if (a->first < 0 || a->recent < 0 || a->first > a->keep || a->recent > a->keep - a->first)
        return fail(FROG_EINVAL, "first %lld, recent %lld, keep %lld: 0 <= first, recent and first + recent <= keep are wanted", (long long)a->first, (long long)a->recent, (long long)a->keep);
    if (a->keep > kMaxRows) return fail(FROG_EUNSUPPORTED, "more than 2^30 pages chosen");
    TRY(check_queries(a->q, a->q_stride, a->batch, a->heads, a->cache, size));
    if (a->batch == 0 || a->keep == 0) return FROG_OK;
    return a->chosen ? FROG_OK : fail(FROG_EINVAL, "chosen is NULL");
}

int check_paged(const frog_attend_paged_t* a) {
    if (!a) return fail(FROG_EINVAL, "arguments are NULL");
    int size = 0;
    TRY(check_type(a->type, &size));
    TRY(check_cache(a->cache, true, false));
    TRY(check_requests(*a));
    TRY(check_heads(a->heads, a->cache.kv_heads, a->cache.d, a->scale, a->cap));
    TRY(check_queries(a->q, a->q_stride, a->batch, a->heads, a->cache, size));
    if (a->num_chosen < 0) return fail(FROG_EINVAL, "negative size");
    if (a->num_chosen > kMaxRows / a->cache.page) return fail(FROG_EUNSUPPORTED, "more than 2^30 rows chosen");
    if (a->batch == 0) return FROG_OK;
    const int64_t rows[2] = {a->batch, a->heads};
    return check_rows("out", a->out, a->out_stride, rows, size);
}

}  // namespace
}  // namespace frog

using namespace frog;

extern "C" {

int frog_cache_write(const frog_cache_write_t* a, void* stream) {
    clear_error();
    TRY(check_write(a));
    return guarded([&] { return launch_cache_write(*a, (hipStream_t)stream); });
}

int frog_cache_read(const frog_cache_read_t* a, void* stream) {
    clear_error();
    TRY(check_read(a));
    return guarded([&] { return launch_cache_read(*a, (hipStream_t)stream); });
}

int64_t frog_select_pages_workspace(const frog_select_pages_t* a) {
    clear_error();
    int rc = check_select(a);
    return rc != FROG_OK ? rc : select_pages_ws(*a);
}

int frog_select_pages(const frog_select_pages_t* a, void* stream) {
    clear_error();
    TRY(check_select(a));
    return guarded([&] { return with_ws(*a, select_pages_ws(*a), (hipStream_t)stream, [&](void* ws) { return launch_select_pages(*a, ws, (hipStream_t)stream); }); });
}

int64_t frog_attend_paged_workspace(const frog_attend_paged_t* a) {
    clear_error();
    int rc = check_paged(a);
    return rc != FROG_OK ? rc : attend_paged_ws(*a);
}

int frog_attend_paged(const frog_attend_paged_t* a, void* stream) {
    clear_error();
    TRY(check_paged(a));
    return guarded([&] { return with_ws(*a, attend_paged_ws(*a), (hipStream_t)stream, [&](void* ws) { return launch_attend_paged(*a, ws, (hipStream_t)stream); }); });
}

}  // extern "C"

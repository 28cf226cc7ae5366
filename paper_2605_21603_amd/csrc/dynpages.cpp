// C entry points of the page operators: checks of the arguments, the plan's place in the workspace, launches.
#include "../../include/dynlayer.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "host_error.h"
#include "pages.h"

namespace {

using dyn::fail;

static_assert((int)DYN_PAGES_DONE == (int)dyn::PAGES_DONE && (int)DYN_PAGES_NONE_LEFT == (int)dyn::PAGES_NONE_LEFT &&
              (int)DYN_PAGES_REFUSED == (int)dyn::PAGES_REFUSED, "answers of a request");

size_t page_bytes(const dyn_page_pool *p) {
    return (size_t)p->n_kv_heads * p->page_size * p->head_dim * (p->dtype == DYN_F32 ? 4 : 2);
}

// The plan of up to n requests on a pool, in 32-bit words behind one another; base NULL: only how many.
size_t plan_words(const dyn_page_pool *p, int n, int32_t *base, dyn::PagesPlan *out) {
    size_t at = 0;
    auto take = [&](size_t words) {
        int32_t *const q = base ? base + at : nullptr;
        at += (words + 63) & ~(size_t)63;
        return q;
    };
    dyn::PagesPlan w;
    w.n_copies = take(1);
    w.owner = take((size_t)p->n_rows);
    w.first = take((size_t)n);
    w.had = take((size_t)n);
    w.has = take((size_t)n);
    w.need = take((size_t)n);
    w.length = take((size_t)n);
    w.src = take((size_t)n);
    const size_t copies = (size_t)std::max(n, p->n_pages);            // compaction moves pages, not requests
    w.copy_src = take(copies);
    w.copy_dst = take(copies);
    w.fresh = take((size_t)p->n_pages);
    if (out) *out = w;
    return at;
}

dyn_status check_geometry(const dyn_page_pool *p) {
    if (!p) return fail(DYN_ERR_INVALID_ARG, "NULL pool");
    if (p->dtype != DYN_F32 && p->dtype != DYN_BF16) return fail(DYN_ERR_INVALID_ARG, "dtype %d", p->dtype);
    if (p->n_layers < 1 || p->n_kv_heads < 1 || p->head_dim < 1 || p->page_size < 1 || p->n_pages < 1 || p->n_rows < 1 || p->max_pages_per_row < 1)
        return fail(DYN_ERR_INVALID_ARG, "non-positive pool dimension");
    if (p->page_size > 512) return fail(DYN_ERR_UNSUPPORTED, "page_size > 512");
    if (page_bytes(p) % 16) return fail(DYN_ERR_UNSUPPORTED, "a page has %zu bytes: no multiple of 16", page_bytes(p));
    if (p->n_pages > 1 << 30 || (long long)p->max_pages_per_row * p->page_size > 0x7fffffffLL)
        return fail(DYN_ERR_UNSUPPORTED, "positions and pages are counted in 32 bits");
    return DYN_OK;
}

dyn_status check_caches(const dyn_page_pool *p) {
    if ((p->k_cache_layers != nullptr) != (p->v_cache_layers != nullptr))
        return fail(DYN_ERR_INVALID_ARG, "k_cache_layers and v_cache_layers go together");
    if (!p->k_cache_layers) {
        if (!p->k_cache || !p->v_cache) return fail(DYN_ERR_INVALID_ARG, "NULL cache pointer");
        if (p->n_layers > 1 && p->kv_layer_stride < page_bytes(p) * p->n_pages)
            return fail(DYN_ERR_INVALID_ARG, "kv_layer_stride %zu is less than a layer's pages", p->kv_layer_stride);
        if (((uintptr_t)p->k_cache | (uintptr_t)p->v_cache | p->kv_layer_stride) & 15) return fail(DYN_ERR_INVALID_ARG, "cache pointer or stride not 16-byte aligned");
        return DYN_OK;
    }
    for (int l = 0; l < p->n_layers; ++l) {
        if (!p->k_cache_layers[l] || !p->v_cache_layers[l]) return fail(DYN_ERR_INVALID_ARG, "layer %d: NULL cache pointer in k_cache_layers / v_cache_layers", l);
        if (((uintptr_t)p->k_cache_layers[l] | (uintptr_t)p->v_cache_layers[l]) & 15) return fail(DYN_ERR_INVALID_ARG, "layer %d: cache pointer not 16-byte aligned", l);
    }
    return DYN_OK;
}

dyn_status check_tables(const dyn_page_pool *p, int n, dyn::PagesPlan *plan) {
    if (!p->block_table || !p->seq_len || !p->ref_count) return fail(DYN_ERR_INVALID_ARG, "NULL table pointer in pool");
    if (!p->workspace || ((uintptr_t)p->workspace & 255)) return fail(DYN_ERR_WORKSPACE, "workspace missing or not 256-byte aligned");
    const size_t need = plan_words(p, n, nullptr, nullptr) * sizeof(int32_t);
    if (p->workspace_bytes < need) return fail(DYN_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu", p->workspace_bytes, need);
    plan_words(p, n, (int32_t *)p->workspace, plan);
    return DYN_OK;
}

dyn::PageTables tables_of(const dyn_page_pool *p) {
    return dyn::PageTables{p->page_size, p->n_pages, p->n_rows, p->max_pages_per_row, p->block_table, p->seq_len, p->ref_count};
}

// Layers l0 .. of the pool, as many as one launch serves.
dyn::PageLayers layers_from(const dyn_page_pool *p, int l0) {
    dyn::PageLayers l{};
    l.n = std::min(p->n_layers - l0, dyn::kPageLayers);
    l.page_bytes = page_bytes(p);
    for (int i = 0; i < l.n; ++i) {
        l.k[i] = p->k_cache_layers ? (char *)p->k_cache_layers[l0 + i] : (char *)p->k_cache + (size_t)(l0 + i) * p->kv_layer_stride;
        l.v[i] = p->v_cache_layers ? (char *)p->v_cache_layers[l0 + i] : (char *)p->v_cache + (size_t)(l0 + i) * p->kv_layer_stride;
    }
    return l;
}

dyn_status launched(hipError_t e, const char *what) {
    return e == hipSuccess ? DYN_OK : fail(DYN_ERR_HIP, "launch of %s failed: %s", what, hipGetErrorString(e));
}

// Plan, then tables with the first layers' copies, then the copies of whatever layers one launch does not hold.
dyn_status plan_and_apply(const dyn_page_pool *p, int what, const char *name, const dyn::PagesPlan &plan, int n, int rows, size_t most_copies, const int32_t *xs,
                          const int32_t *ys, int32_t *status, int32_t *new_page, int32_t *n_live, hipStream_t s) {
    const dyn::PageTables t = tables_of(p);
    hipError_t e = dyn::launch_pages_plan(what, t, plan, n, xs, ys, status, new_page, n_live, s);
    if (e == hipSuccess) e = dyn::launch_pages_apply(what, t, plan, layers_from(p, 0), rows, most_copies, xs, ys, new_page, s);
    for (int l0 = dyn::kPageLayers; l0 < p->n_layers && e == hipSuccess; l0 += dyn::kPageLayers)
        e = dyn::launch_pages_copy(what == dyn::PAGES_COMPACT, layers_from(p, l0), p->n_pages, (int)most_copies, plan.copy_src, plan.copy_dst, plan.n_copies, s);
    return launched(e, name);
}

}  // namespace

extern "C" {

size_t dyn_pages_workspace_bytes(const dyn_page_pool *p, int max_requests) {
    if (max_requests < 0 || check_geometry(p) != DYN_OK) return 0;
    return plan_words(p, max_requests, nullptr, nullptr) * sizeof(int32_t);
}

dyn_status dyn_pages_copy(const dyn_page_pool *p, int n, const int32_t *src, const int32_t *dst, void *hip_stream) {
    dyn_status rc = check_geometry(p);
    if (rc != DYN_OK || (rc = check_caches(p)) != DYN_OK) return rc;
    if (n < 0) return fail(DYN_ERR_INVALID_ARG, "negative number of pages");
    if (n == 0) return DYN_OK;
    if (!src || !dst) return fail(DYN_ERR_INVALID_ARG, "NULL argument");
    for (int l0 = 0; l0 < p->n_layers && rc == DYN_OK; l0 += dyn::kPageLayers)
        rc = launched(dyn::launch_pages_copy(true, layers_from(p, l0), p->n_pages, n, src, dst, nullptr, (hipStream_t)hip_stream), "page copy");
    return rc;
}

dyn_status dyn_pages_fork(const dyn_page_pool *p, int n, const int32_t *parent, const int32_t *child, int32_t *status, void *hip_stream) {
    dyn::PagesPlan plan;
    dyn_status rc = check_geometry(p);
    if (rc != DYN_OK || (rc = check_caches(p)) != DYN_OK) return rc;
    if (n < 0) return fail(DYN_ERR_INVALID_ARG, "negative number of requests");
    if ((rc = check_tables(p, n, &plan)) != DYN_OK || n == 0) return rc;
    if (!parent || !child || !status) return fail(DYN_ERR_INVALID_ARG, "NULL argument");
    return plan_and_apply(p, dyn::PAGES_FORK, "fork", plan, n, n, (size_t)n, parent, child, status, nullptr, nullptr, (hipStream_t)hip_stream);
}

dyn_status dyn_pages_resize(const dyn_page_pool *p, int n, const int32_t *row, const int32_t *length, int32_t *status, void *hip_stream) {
    dyn::PagesPlan plan;
    dyn_status rc = check_geometry(p);
    if (rc != DYN_OK || (rc = check_caches(p)) != DYN_OK) return rc;
    if (n < 0) return fail(DYN_ERR_INVALID_ARG, "negative number of requests");
    if ((rc = check_tables(p, n, &plan)) != DYN_OK || n == 0) return rc;
    if (!row || !length || !status) return fail(DYN_ERR_INVALID_ARG, "NULL argument");
    return plan_and_apply(p, dyn::PAGES_RESIZE, "resize", plan, n, n, (size_t)n, row, length, status, nullptr, nullptr, (hipStream_t)hip_stream);
}

dyn_status dyn_pages_compact(const dyn_page_pool *p, int32_t *new_page, int32_t *n_live, void *hip_stream) {
    dyn::PagesPlan plan;
    dyn_status rc = check_geometry(p);
    if (rc != DYN_OK || (rc = check_caches(p)) != DYN_OK || (rc = check_tables(p, 0, &plan)) != DYN_OK) return rc;
    if (!new_page || !n_live) return fail(DYN_ERR_INVALID_ARG, "NULL argument");
    return plan_and_apply(p, dyn::PAGES_COMPACT, "compaction", plan, 0, p->n_rows, (size_t)p->n_pages / 2, nullptr, nullptr, nullptr, new_page, n_live,
                          (hipStream_t)hip_stream);
}

}  // extern "C"

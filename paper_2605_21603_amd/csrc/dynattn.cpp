// C entry points of the attention over shared prefixes: checks of the arguments, the workspace, the launch.
#include "../../include/dynlayer.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_shared.h"
#include "host_error.h"
#include "kernels.h"

namespace {

using dyn::fail;

struct Layout { size_t part_o, part_ml, plan, total; };

size_t align_up(size_t v) { return (v + 255) & ~(size_t)255; }

dyn_status check_sizes(const dyn_attn_batch *b) {
    if (!b) return fail(DYN_ERR_INVALID_ARG, "NULL batch");
    if (b->dtype != DYN_F32 && b->dtype != DYN_BF16) return fail(DYN_ERR_INVALID_ARG, "dtype %d", b->dtype);
    if (b->n_q_heads < 1 || b->n_kv_heads < 1 || b->head_dim < 1 || b->page_size < 1) return fail(DYN_ERR_INVALID_ARG, "non-positive attention dimension");
    if (b->n_q_heads % b->n_kv_heads) return fail(DYN_ERR_INVALID_ARG, "n_q_heads not a multiple of n_kv_heads");
    const int d = b->head_dim;
    if (d < 8 || d > 2 * dyn::kMaxHalfDim || (d & (d - 1))) return fail(DYN_ERR_UNSUPPORTED, "head_dim must be a power of two in 8..256");
    if (b->page_size > 512) return fail(DYN_ERR_UNSUPPORTED, "page_size > 512");
    if ((long long)b->n_q_heads * d > 0x7fffffffLL) return fail(DYN_ERR_UNSUPPORTED, "rows of %lld elements", (long long)b->n_q_heads * d);
    if (b->kv_chunk_positions != 0 && (b->kv_chunk_positions < 64 || b->kv_chunk_positions > 65536 || b->kv_chunk_positions % b->page_size))
        return fail(DYN_ERR_INVALID_ARG, "kv_chunk_positions = %d: 0, or a multiple of page_size in 64..65536", b->kv_chunk_positions);
    if (b->n_tokens < 0 || b->n_seqs < 0) return fail(DYN_ERR_INVALID_ARG, "negative n_tokens or n_seqs");
    if (b->n_tokens >= 1 << 24) return fail(DYN_ERR_UNSUPPORTED, "%d tokens", b->n_tokens);
    if (b->n_tokens > 0 && (b->n_seqs < 1 || b->max_pages_per_seq < 1)) return fail(DYN_ERR_INVALID_ARG, "tokens without sequences or pages");
    if ((long long)b->n_seqs * b->max_pages_per_seq >= 1 << 29) return fail(DYN_ERR_UNSUPPORTED, "block table of 2^29 entries or more");
    if ((long long)b->max_pages_per_seq * b->page_size > 1 << 30) return fail(DYN_ERR_UNSUPPORTED, "sequences of more than 2^30 positions");
    return DYN_OK;
}

// The shape as the layer has it (dynlayer.cpp, tensor_sizes), and where the call's scratch lies.
dyn::AttnShape shape_of(const dyn_attn_batch *b, dyn::AttnPrefix *prefix, Layout *w) {
    const int pages = std::max(b->max_pages_per_seq, 1), chunk = std::max(1, (b->kv_chunk_positions ? b->kv_chunk_positions : 256) / b->page_size);
    dyn::AttnShape sh{b->n_q_heads, b->n_kv_heads, b->head_dim, b->page_size, pages, chunk, (pages + chunk - 1) / chunk, 0};
    sh.max_chunks = dyn::attn_own_max_chunks(b->dtype, sh);
    *prefix = dyn::AttnPrefix{b->prefix_lead, b->prefix_pages, b->n_seqs, dyn::attn_prefix_max_chunks(b->dtype, sh), b->seq_of_token, b->pos_of_token, b->n_tokens};
    const size_t partials = (size_t)b->n_tokens * b->n_q_heads * (sh.max_chunks + prefix->max_chunks);
    w->part_o = 0;
    w->part_ml = align_up(partials * b->head_dim * sizeof(float));
    w->plan = w->part_ml + align_up(partials * 2 * sizeof(float));
    w->total = w->plan + align_up(dyn::attn_shared_plan_words(sh, *prefix, b->n_tokens) * sizeof(int32_t));
    return sh;
}

}  // namespace

extern "C" {

size_t dyn_attn_shared_workspace_bytes(const dyn_attn_batch *b) {
    if (check_sizes(b) != DYN_OK) return 0;
    dyn::AttnPrefix prefix;
    Layout w;
    shape_of(b, &prefix, &w);
    return w.total;
}

dyn_status dyn_attn_shared(const dyn_attn_batch *b, void *hip_stream) {
    dyn_status rc = check_sizes(b);
    if (rc != DYN_OK) return rc;
    if (b->n_tokens == 0) return DYN_OK;
    if (!b->q || !b->out || !b->seq_of_token || !b->pos_of_token || !b->block_table || !b->k_cache || !b->v_cache)
        return fail(DYN_ERR_INVALID_ARG, "NULL tensor pointer in batch");
    if (b->q == b->out) return fail(DYN_ERR_INVALID_ARG, "out must not alias q");
    if ((b->prefix_lead != nullptr) != (b->prefix_pages != nullptr)) return fail(DYN_ERR_INVALID_ARG, "prefix_lead and prefix_pages go together");
    const int width = b->n_q_heads * b->head_dim, vec = b->dtype == DYN_F32 ? 4 : 8;
    if (b->ld_q < width || b->ld_out < width) return fail(DYN_ERR_INVALID_ARG, "rows of %d elements do not fit ld_q = %d or ld_out = %d", width, b->ld_q, b->ld_out);
    if (((uintptr_t)b->q | (uintptr_t)b->out | (uintptr_t)b->k_cache | (uintptr_t)b->v_cache) & 15 || b->ld_q % vec || b->ld_out % vec)
        return fail(DYN_ERR_INVALID_ARG, "q, out and the caches need 16-byte aligned rows");
    dyn::AttnPrefix prefix;
    Layout w;
    const dyn::AttnShape sh = shape_of(b, &prefix, &w);
    if (!b->workspace || ((uintptr_t)b->workspace & 255)) return fail(DYN_ERR_WORKSPACE, "workspace missing or not 256-byte aligned");
    if (b->workspace_bytes < w.total) return fail(DYN_ERR_WORKSPACE, "workspace has %zu bytes, this batch needs %zu", b->workspace_bytes, w.total);
    char *const base = (char *)b->workspace;
    const hipError_t e = dyn::launch_attention_shared(b->dtype, b->q, b->ld_q, b->seq_of_token, b->pos_of_token, b->block_table, b->k_cache, b->v_cache, b->out, b->ld_out,
                                                      (float *)(base + w.part_o), (float *)(base + w.part_ml), (int32_t *)(base + w.plan), sh, prefix,
                                                      b->n_tokens, (hipStream_t)hip_stream, nullptr, nullptr, 0);
    if (e != hipSuccess) return fail(DYN_ERR_HIP, "launch of the attention failed: %s", hipGetErrorString(e));
    return DYN_OK;
}

}  // extern "C"

// Attention over shared prefixes: what its host side (dynattn.cpp, dynlayer.cpp) and kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "attn_shape.h"

namespace dyn {

// What the sequences of a batch share: sequence s reads the first pages[s] pages of its row together with every
// other sequence whose lead is lead[s].  Null: nothing is shared.
struct AttnPrefix {
    const int32_t *lead = nullptr, *pages = nullptr;
    int n_seqs = 0;
    int max_chunks = 0;          // the most chunks a token's shared keys can have; its own ones are AttnShape::max_chunks
    const int32_t *seq_of_token = nullptr, *pos_of_token = nullptr;   // all rows of the batch, of which a call may serve some
    int rows = 0;
};

// The most chunks of a row's shared and of its own keys, of a batch whose rows have sh.max_pages_per_seq pages at most.
int attn_prefix_max_chunks(int dtype, const AttnShape &sh);
int attn_own_max_chunks(int dtype, const AttnShape &sh);
// 32-bit words of scratch for `rows` rows; sh.max_chunks: of the rows' own keys.
size_t attn_shared_plan_words(const AttnShape &sh, const AttnPrefix &prefix, int rows);
// As launch_attention, with q rows ld_q elements apart, part_o [rows, sh.max_chunks + prefix.max_chunks, n_q, head_dim] and part_ml to match; a row of position -1 attends
// nothing and its output is zero.  layer: of the step; from layer 1 on `plan` holds what layer 0's call on the same rows left.
hipError_t launch_attention_shared(int dtype, const void *q, int ld_q, const int32_t *seq_of_token, const int32_t *pos_of_token, const int32_t *block_table,
                                   const void *k_cache, const void *v_cache, void *out, int ld_out, float *part_o, float *part_ml, int32_t *plan,
                                   const AttnShape &sh, const AttnPrefix &prefix, int rows, hipStream_t s, hipEvent_t mid, hipEvent_t pre, int layer);

}  // namespace dyn

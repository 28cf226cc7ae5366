// The plan of an attention over shared prefixes: where its arrays and lists lie, and the launch that fills them (kernels_attn_shared_plan.hip).
#pragma once
#include "attn_shared.h"
#include "kernels.h"

namespace dyn {

// How rows of a shape are attended: by the forms of this operator (bf16, 128-wide heads), by the layer's general one on the matrix
// cores (attn_tile), or by its plain loops, without sharing.
enum AttnForm { SHARE_LISTS = 0, SHARE_TILES = 1, SHARE_NOTHING = 2 };

struct SharedPlan {
    // Per row; p_: of its shared keys, s_: of its own.  seq: offset into the block table, pos: the last key (-1: none), ct: positions
    // per chunk.
    int32_t *p_seq, *p_pos, *p_ct, *s_seq, *s_pos, *s_ct;
    // Work lists, [0] = entries, entry i at 2 + 2 i: the first token row, then chunk | tokens << 20.  items: up to 16 columns (a token and a q head
    // each) of shared keys, or the own keys of a sequence's tokens (kOwnItem set in the row).  p_blocks, s_blocks: query blocks of shared and
    // of own keys.  [1] = a counter that entries are claimed from.
    int32_t *items, *p_blocks, *s_blocks;
    // What the lists take, in us of one CU and kv head: [0] the items, [1] the query blocks.
    float *cost;
};
constexpr int kOwnItem = 1 << 30;

SharedPlan attn_shared_plan(int32_t *plan, const AttnShape &sh, const AttnPrefix &prefix, int rows);
AttnForm attn_shared_form(int dtype, const AttnShape &sh, const void *k_cache, const void *v_cache);
hipError_t launch_attn_shared_plan(AttnForm form, const int32_t *seq_of_token, const int32_t *pos_of_token, const AttnShape &sh, const AttnPrefix &prefix, int rows,
                                   const SharedPlan &w, hipStream_t s);

// kernels_attn_generic.hip: what the general form takes (of shapes, and of caches too); its launch over the plan's lists; and the plain loops' over rows
bool attn_tile_shape(const AttnShape &sh);
bool attn_tile_takes(const AttnShape &sh, const void *k_cache, const void *v_cache);
hipError_t launch_attention_parts(int dtype, const void *q, int ld_q, const int32_t *block_table, const void *k_cache, const void *v_cache, float *part_o, float *part_ml,
                                  const AttnShape &sh, const SharedPlan &w, int shared_slots, int rows, hipStream_t s);
hipError_t launch_attention_own(int dtype, const void *q, int ld_q, const int32_t *seq_of_token, const int32_t *pos_of_token, const int32_t *block_table, const void *k_cache,
                                const void *v_cache, float *part_o, float *part_ml, const AttnShape &sh, int rows, hipStream_t s);

}  // namespace dyn

// The plan of an attention over shared prefixes (kernels_attn_shared.hip), built on the device from the step's arrays.
//
// Every row's keys are cut in two: the shared ones, which it attends together with the rows around it that share the same, and its
// own.  Each half is described by arrays that take the place of the batch's (an offset into the block table for the
// sequence, the last key for the position), and work lists name what exists of it.  Who shares with a row, and how long chunks are, is counted
// over the whole batch and not over the dispatch, so a row's sums do not depend on the schedule.  A row that stands inside the shared positions, alone with its lead or outside the table attends all its keys as its own.
// One workgroup of 16 waves walks the rows 1024 at a time, twice: first the runs of rows that share the same, then what each leads.
#include <algorithm>

#include "attn_shared_plan.h"
#include "common.h"

namespace dyn {

int attn_prefill_block_tokens(const AttnShape &sh);

namespace {

constexpr int kShareSeqs = 8192;              // sequences whose leads are counted in LDS; a batch of more attends without sharing
// Up to kFewSharers sets of 16 columns (a token and a q head each) of a prefix are served like decodes, K and V read once per set; more by query
// blocks, which read them once for all.
constexpr int kFewSharers = 2;

template <class Combine>
__device__ __forceinline__ int scan_wave(int x, Combine &&combine) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off, 64);
        if (lane >= off) x = combine(x, y);
    }
    return x;
}
__device__ __forceinline__ int add(int a, int b) { return a + b; }
__device__ __forceinline__ int larger(int a, int b) { return a > b ? a : b; }

struct PlanRule {
    int tg_many, tg_few, most_few;      // tokens of a query block and of an item; the most tokens of a prefix that items serve
    int most_positions;                 // the longest chunk of a single token's own keys
};

// Chunks, from the batch: `shared` = keys of a prefix times query blocks that attend it, summed over the prefixes; `own` = keys of single
// tokens, summed.  A chunk costs a partial set per column, written and read again, and too few of them leave CUs idle.
// Query blocks: what gives every CU a piece, or, beside single tokens' keys, what takes half as long as those (a tile of 64 positions
// some 4 us, keys of one kv head 512 bytes at 5.5 TB/s); two tiles at least, and at most 32 chunks a prefix.
__device__ __forceinline__ int block_positions(long long shared, long long own, int n_kv, int keys) {
    const long long want = max(max(shared * n_kv / 256, own * n_kv * 3 / 4096), (long long)keys / 32);
    return (int)min(max((want + 63) / 64 * 64, 128ll), 8192ll);
}
// Items: four rounds of the chip's 2048 waves, at least 64 positions and at most 64 chunks a token.
__device__ __forceinline__ int item_positions(long long own, int n_kv, int most, int keys) {
    const long long want = min(max((own * n_kv / 8192 + 63) / 64 * 64, 64ll), (long long)most);
    return (int)max(want, ((long long)keys / 64 + 63) / 64 * 64);
}

template <AttnForm FORM>
__global__ __launch_bounds__(1024) void attn_shared_plan_kernel(const int32_t *seq_of_token, const int32_t *pos_of_token, int rows, AttnPrefix prefix, AttnShape sh,
                                                                PlanRule rule, SharedPlan w) {
    __shared__ int members[FORM == SHARE_NOTHING ? 1 : kShareSeqs];
    __shared__ int sums[3][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ps = sh.page_size, max_pages = sh.max_pages_per_seq;
    const bool any = FORM != SHARE_NOTHING && prefix.lead != nullptr;
    auto shares = [&](int s, int &lead, int &pages) {                // sequence s names a lead and pages of its row
        if (!any || s < 0 || s >= prefix.n_seqs) return false;
        lead = prefix.lead[s];
        pages = prefix.pages[s];
        return lead >= 0 && lead < prefix.n_seqs && pages >= 1 && pages < max_pages;
    };
    struct Row { int seq, pos, lead, keys; };                        // lead -1: shares nothing
    auto row_of = [&](int seq, int pos) {
        Row r{seq, pos, -1, 0};
        int lead, pages;
        if (pos >= 0 && shares(seq, lead, pages) && pos >= pages * ps && members[lead] >= 0) { r.lead = lead; r.keys = pages * ps; }
        return r;
    };
    // members: sequences that name the lead; then, of those named by two and more, the batch's tokens behind the prefix, others -1
    __shared__ long long batch[2];                                   // keys of shared prefixes over tokens, own keys of single tokens
    if (threadIdx.x < 2) batch[threadIdx.x] = 0;
    if (any) {
        for (int s = threadIdx.x; s < prefix.n_seqs; s += 1024) members[s] = 0;
        __syncthreads();
        for (int s = threadIdx.x; s < prefix.n_seqs; s += 1024) {
            int lead, pages;
            if (shares(s, lead, pages)) atomicAdd(&members[lead], 1);
        }
        __syncthreads();
        for (int s = threadIdx.x; s < prefix.n_seqs; s += 1024) members[s] = members[s] > 1 ? 0 : -1;
    }
    __syncthreads();
    if constexpr (FORM != SHARE_NOTHING) {
        long long shared = 0, own = 0;
        for (int t = threadIdx.x; t < prefix.rows; t += 1024) {
            const int seq = prefix.seq_of_token[t];
            const bool single = (t == 0 || prefix.seq_of_token[t - 1] != seq) && (t + 1 >= prefix.rows || prefix.seq_of_token[t + 1] != seq);
            const Row r = row_of(seq, prefix.pos_of_token[t]);
            if (r.lead >= 0) {
                atomicAdd(&members[r.lead], 1);
                shared += r.keys;
            }
            if (single) own += r.pos + 1 - r.keys;
        }
        if (__any(shared || own)) {
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) { shared += __shfl_xor(shared, off, 64); own += __shfl_xor(own, off, 64); }
            if (lane == 0) {
                atomicAdd((unsigned long long *)&batch[0], (unsigned long long)shared);
                atomicAdd((unsigned long long *)&batch[1], (unsigned long long)own);
            }
        }
        __syncthreads();
    }
    const long long batch_shared = batch[0] / rule.tg_many, batch_own = batch[1];
    int run_before = -1, blocks_before = 0;                          // the last run's first row, and the query blocks, before these rows
    for (int t0 = 0; t0 < rows; t0 += 1024) {
        const int t = t0 + (int)threadIdx.x;
        Row r{-1, -1, -1, 0};
        bool starts = false;
        if (t < rows) {
            const int prev = max(t - 1, 0);
            r = row_of(seq_of_token[t], pos_of_token[t]);
            const Row before = row_of(seq_of_token[prev], pos_of_token[prev]);
            starts = r.lead >= 0 && (t == 0 || before.lead != r.lead || before.keys != r.keys);
        }
        int run = scan_wave(starts ? t : -1, larger);                // the latest start up to here
        if (lane == 63) sums[0][wave] = run;
        __syncthreads();
        run = max(run, run_before);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            if (k < wave) run = max(run, sums[0][k]);
            run_before = max(run_before, sums[0][k]);
        }
        const bool few = r.lead >= 0 && members[r.lead] <= rule.most_few;
        const int width = few ? rule.tg_few : rule.tg_many;
        const bool leads = r.lead >= 0 && (t - run) % width == 0;
        int blocks = 0;
        if constexpr (FORM == SHARE_TILES) {
            const unsigned long long mask = __ballot(leads);
            if (lane == 0) sums[1][wave] = __popcll(mask);
            __syncthreads();
            blocks = blocks_before + __popcll(mask & ((2ull << lane) - 1));
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                if (k < wave) blocks += sums[1][k];
                blocks_before += sums[1][k];
            }
        }
        if (t < rows) {
            const bool on = r.lead >= 0;
            w.s_seq[t] = r.pos < 0 ? -1 - t : r.seq * max_pages + r.keys / ps;
            w.s_pos[t] = r.pos < 0 ? -1 : r.pos - r.keys;
            w.p_pos[t] = on ? r.keys - 1 : -1;
            if constexpr (FORM == SHARE_LISTS) {
                w.p_seq[t] = on ? r.lead * max_pages : -1;
                w.p_ct[t] = !on ? 64 : few ? item_positions(batch_own, sh.n_kv, rule.most_positions, 2 * r.keys)
                                           : block_positions(batch_shared, batch_own, sh.n_kv, r.keys);
                w.run[t] = on ? run : -1 - t;
                w.width[t] = leads ? (few ? -width : width) : 0;
            } else {
                w.p_seq[t] = on ? (r.lead * max_pages) | (few ? kTileNarrow : kTileWide) | (int)((unsigned)blocks << 31) : -1;
            }
        }
        __syncthreads();
    }
    if constexpr (FORM == SHARE_LISTS) {
        __threadfence_block();
        __syncthreads();
        int entries[3] = {0, 0, 0};                                  // of items, p_blocks, s_blocks
        float cost[2] = {0.f, 0.f};
        __shared__ float costs[2][16];
        for (int t0 = 0; t0 < rows; t0 += 1024) {
            const int t = t0 + (int)threadIdx.x;
            int p_tok = 0, p_n = 0, s_tok = 0, s_n = 0;              // what row t leads: tokens and chunks
            bool few = false, single = false;
            if (t < rows) {
                const int width = w.width[t], s = w.s_seq[t], p = w.s_pos[t];
                if (width) {
                    few = width < 0;
                    const int run = w.run[t], ct = w.p_ct[t];
                    int lo = 1, hi = min(few ? -width : width, rows - t);
                    if (w.run[t + hi - 1] == run) lo = hi;           // rows t .. t + lo - 1 are of the run
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) >> 1;
                        if (w.run[t + mid - 1] == run) lo = mid;
                        else hi = mid - 1;
                    }
                    p_tok = lo;
                    p_n = (w.p_pos[t] + ct) / ct;
                }
                const bool prev_same = t > 0 && w.s_seq[t - 1] == s, next_same = t + 1 < rows && w.s_seq[t + 1] == s;
                single = !prev_same && !next_same;
                const int tg = rule.tg_many, ct = single ? item_positions(batch_own, sh.n_kv, rule.most_positions, p + 1) : prefill_chunk_positions((p / tg + 1) * tg);
                w.s_ct[t] = ct;
                if (p >= 0 && (single || !prev_same || p % tg == 0)) {
                    int lo = 1, hi = single ? 1 : min(tg - p % tg, rows - t);
                    if (w.s_seq[t + hi - 1] == s) lo = hi;           // positions left in the aligned block that are rows of the sequence
                    while (lo < hi) {
                        const int mid = (lo + hi + 1) >> 1;
                        if (w.s_seq[t + mid - 1] == s) lo = mid;
                        else hi = mid - 1;
                    }
                    s_tok = lo;
                    s_n = (p + s_tok - 1 + ct) / ct;                 // chunks the block's last token reaches
                }
            }
            // a position of an item 512 bytes at 19.5 GB/s, a query block's tile of 64 positions 2 us for its loads and up to 4 for its products
            const float per_block = 2.f / 64, per_token = 4.f / (64 * rule.tg_many);
            if (p_n) (few ? cost[0] : cost[1]) += (w.p_pos[t] + 1) * (few ? 0.026f : per_block + p_tok * per_token);
            if (s_n) (single ? cost[0] : cost[1]) += (w.s_pos[t] + s_tok) * (single ? 0.026f : per_block + s_tok * per_token);
            const int mine[3] = {(few ? p_n : 0) + (single ? s_n : 0), few ? 0 : p_n, single ? 0 : s_n};
            int start[3];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int incl = scan_wave(mine[k], add);
                if (lane == 63) sums[k][wave] = incl;
                start[k] = entries[k] + incl - mine[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (j < wave) start[k] += sums[k][j];
                    entries[k] += sums[k][j];
                }
            __syncthreads();
            int32_t *at = few ? w.items + 2 + 2 * (size_t)start[0] : w.p_blocks + 2 + 2 * (size_t)start[1];
            for (int c = 0; c < p_n; ++c) { *at++ = t; *at++ = c | (p_tok << 20); }
            at = single ? w.items + 2 + 2 * (size_t)(start[0] + (few ? p_n : 0)) : w.s_blocks + 2 + 2 * (size_t)start[2];
            for (int c = 0; c < s_n; ++c) { *at++ = single ? t | kOwnItem : t; *at++ = c | (s_tok << 20); }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float x = wave_sum(cost[k]);
            if (lane == 0) costs[k][wave] = x;
        }
        __syncthreads();
        if (threadIdx.x < 2) {
            float x = 0.f;
            for (int j = 0; j < 16; ++j) x += costs[threadIdx.x][j];
            w.cost[threadIdx.x] = x;
        }
        if (threadIdx.x == 0) {
            w.items[0] = entries[0];
            w.p_blocks[0] = entries[1];
            w.s_blocks[0] = entries[2];
            w.p_blocks[1] = w.s_blocks[1] = 0;
        }
    }
}

}  // namespace

int attn_prefix_max_chunks(int dtype, const AttnShape &sh) {
    const long positions = (long)sh.max_pages_per_seq * sh.page_size;
    if (!attention_mfma_supported(dtype, sh)) return (sh.max_pages_per_seq + sh.chunk_pages - 1) / sh.chunk_pages;
    const long most = std::max<long>(32, (positions + 8191) / 8192);
    return (int)std::max<long>(1, std::min<long>(most, (positions + 63) / 64));
}

int attn_own_max_chunks(int dtype, const AttnShape &sh) {
    const int chunks = (sh.max_pages_per_seq + sh.chunk_pages - 1) / sh.chunk_pages;
    if (!attention_mfma_supported(dtype, sh)) return chunks;
    const long positions = (long)sh.max_pages_per_seq * sh.page_size;
    const int items = std::max(chunks, (int)std::min<long>(64, (positions + 63) / 64));
    return std::max(items, attn_prefill_max_chunks(positions));
}

size_t attn_shared_plan_words(const AttnShape &sh, const AttnPrefix &prefix, int rows) {
    const size_t own = (size_t)sh.max_chunks * rows, shared = (size_t)prefix.max_chunks * rows;
    return (size_t)rows * 8 + 8 + 4 * (own + shared);          // (for rows together no more than for each of them alone)
}

SharedPlan attn_shared_plan(int32_t *plan, const AttnShape &sh, const AttnPrefix &prefix, int rows) {
    SharedPlan w;
    int32_t *at = plan;
    for (int32_t **a : {&w.p_seq, &w.p_pos, &w.p_ct, &w.s_seq, &w.s_pos, &w.s_ct, &w.run, &w.width}) { *a = at; at += rows; }
    const size_t own = (size_t)sh.max_chunks * rows, shared = (size_t)prefix.max_chunks * rows;
    w.cost = (float *)at;
    w.items = at + 2;
    w.p_blocks = w.items + 2 + 2 * (own + shared);
    w.s_blocks = w.p_blocks + 2 + 2 * shared;
    return w;
}

AttnForm attn_shared_form(int dtype, const AttnShape &sh, const void *k_cache, const void *v_cache) {
    return attention_mfma_supported(dtype, sh) ? SHARE_LISTS : attn_tile_takes(sh, k_cache, v_cache) ? SHARE_TILES : SHARE_NOTHING;
}

hipError_t launch_attn_shared_plan(AttnForm form, const int32_t *seq_of_token, const int32_t *pos_of_token, const AttnShape &sh, const AttnPrefix &prefix, int rows,
                                   const SharedPlan &w, hipStream_t s) {
    const int G = sh.n_q / sh.n_kv, TG = G <= 16 ? 16 / G : 1;
    AttnPrefix p = prefix;
    if (p.n_seqs > kShareSeqs) p.lead = nullptr;
    const dim3 one(1), block(1024);
    if (form == SHARE_LISTS) {
        const PlanRule rule{attn_prefill_block_tokens(sh), TG, kFewSharers * TG, sh.chunk_pages * sh.page_size};
        hipLaunchKernelGGL(attn_shared_plan_kernel<SHARE_LISTS>, one, block, 0, s, seq_of_token, pos_of_token, rows, p, sh, rule, w);
    } else if (form == SHARE_TILES) {
        hipLaunchKernelGGL(attn_shared_plan_kernel<SHARE_TILES>, one, block, 0, s, seq_of_token, pos_of_token, rows, p, sh, PlanRule{4 * TG, TG, TG, 0}, w);
    } else {
        hipLaunchKernelGGL(attn_shared_plan_kernel<SHARE_NOTHING>, one, block, 0, s, seq_of_token, pos_of_token, rows, p, sh, PlanRule{1, 1, 0, 0}, w);
    }
    return hipGetLastError();
}

}  // namespace dyn

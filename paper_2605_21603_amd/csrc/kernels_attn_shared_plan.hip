// The plan of an attention over shared prefixes (kernels_attn_shared.hip), built on the device from the step's arrays.
//
// Every row's keys are cut in two: the shared ones, which it attends together with the rows around it that share the same, and its
// own.  Each half is described by arrays that take the place of the batch's (an offset into the block table for the
// sequence, the last key for the position), and work lists name what exists of it.  Who shares with a row, and how long chunks are, is counted
// over the whole batch and not over the dispatch, so a row's sums do not depend on the schedule.  A row that stands inside the shared positions, alone with its lead or outside the table attends all its keys as its own.
// What it costs is the latency of its loads, so everything that is looked at twice is kept in LDS: leads and pages of all sequences, and
// which rows go on with the row before them.  5 rows 5.2 us, 256 rows of 256 sequences 6.6, 1563 of 12 sequences 13, 5387 of 242 sequences 29 (a round of 1024 rows 4).
#include <algorithm>

#include "attn_shared_plan.h"
#include "common.h"

namespace dyn {

int attn_prefill_block_tokens(const AttnShape &sh);

namespace {

constexpr int kShareSeqs = 4096;              // sequences whose leads are counted in LDS; a batch of more attends without sharing

// Inclusive scans over the 64 lanes of a wave on the vector ALU (a shuffle goes through LDS).
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x, int empty) { return __builtin_amdgcn_update_dpp(empty, x, CTRL, ROWS, 0xf, false); }
template <class Op>
__device__ __forceinline__ int scan_wave(int x, int empty, Op &&op) {
    x = op(x, moved<0x111, 0xf>(x, empty));      // row_shr 1, 2, 4, 8
    x = op(x, moved<0x112, 0xf>(x, empty));
    x = op(x, moved<0x114, 0xf>(x, empty));
    x = op(x, moved<0x118, 0xf>(x, empty));
    x = op(x, moved<0x142, 0xa>(x, empty));      // row_bcast 15: rows 1 and 3 take the row below's last
    return op(x, moved<0x143, 0xc>(x, empty));   // row_bcast 31: rows 2 and 3 take lane 31's
}
__device__ __forceinline__ int sum_up(int x) { return scan_wave(x, 0, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int sum_all(int x) { return __builtin_amdgcn_readlane(sum_up(x), 63); }

struct PlanRule {
    int tg_many, tg_few;                // tokens of a query block and of an item
    unsigned many_magic, few_magic;     // ceil(2^32 / .)
    int ahead;                          // words of 64 rows that a query block takes
    int short_tokens;                   // a sequence of no more tokens than this in the step is served by items: a set of columns, which waves anywhere take
                                        // (64 of 2 to 8 tokens, 512 to 2048 keys of their own: 116 us with one alone, 112 so, 131 with up to two sets, which read their keys twice)
    int most_positions;                 // the longest chunk of an item's own keys
    int least, least_long;              // the shortest chunk of an item; and where there are two rounds of such
    int n_kv;
    bool tiles;                         // SHARE_TILES
};

// Chunks, from the batch, in sub-tiles of 16 positions: `shared` = keys of a prefix times query blocks that attend it, summed over the
// prefixes; `own` = sequences' own keys, summed.  A chunk costs a partial set per column, written and read again, and too few of them
// leave CUs idle.  Query blocks: what gives three of four CUs (general form: one of four workgroups to a CU) a piece, so that
// rounding leaves no second round of a few (256 tokens on 4 prefixes of 4096 to 8192, a piece for every CU: 77 us, so 64), or, beside items, what takes as long as those (a tile
// of 64 positions some 2 us, keys of one kv head 512 bytes at 5 TB/s; in a third and a half of that, 64 tokens behind 2048 positions took 65 and 59 us and now take 60,
// 256 behind 4 prefixes 275, 272 and 267, 64 of 4 drafts 97, 75 and 76, 256 of them 200, 192 and 187); two tiles at least, and at most 32 chunks a prefix.
// All chunks of a prefix are then of one length, as a short last one would cost nearly all that a chunk does: as many as asked for (12 prompts of 33 to 300 tokens behind
// 4096 keys: 202 -> 176 us), or, where query blocks have the chip to themselves, one fewer if that makes them at most half as long again (166 us; beside
// items it delays the end, 256 tokens behind 4 prefixes 276 -> 295 us).
__device__ __forceinline__ int block_positions(const PlanRule &rule, long long shared, long long own, int keys) {
    const long long want = max(rule.tiles ? shared * rule.n_kv / 64 : max(shared * rule.n_kv / 12, own * rule.n_kv * 3 / 64), ((long long)keys + 31) / 32);
    const int ct = (int)min(max((want + 63) / 64 * 64, 128ll), 8192ll), n = max((keys + (shared > 8 * own && !rule.tiles ? ct / 2 : ct - 1)) / ct, (keys + 8191) / 8192);
    return ((keys + n - 1) / n + 63) / 64 * 64;
}
// Items: four rounds of the chip's 2048 waves (general form: one of 1024 workgroups), at least 64 positions, or 128 where those are two rounds (64 tokens of 16 to 1024
// keys of their own beside 8 alone: 50.0 -> 47.5 us; but pages of 64 positions, 192 tokens of 3 to 584 keys: 98.5 -> 102.5, so 64 there; general form: 128), and at
// most 64 chunks a token.
__device__ __forceinline__ int item_positions(const PlanRule &rule, long long own, int keys) {
    const long long want = own * rule.n_kv / (rule.tiles ? 64 : 512), least = own * rule.n_kv >= 16384 ? rule.least_long : rule.least;
    return (int)max(min(max((want + 63) / 64 * 64, least), (long long)rule.most_positions), ((long long)keys + 4095) / 4096 * 64);
}

// Whether a prefix that `tokens` tokens attend is served by items, which read K and V once for every tg_few of them, and not by query blocks, which read
// them once for all.  In time of a CU, a position of an item takes some 17 ns, of a query block 15 ns, and 10 us around a block and chunk, in which all of
// the CU waits for its claim, its pages, its first tile and its stores: items where they are no more than that, and all by items where the batch's
// would take the chip no longer than a block's 14 us.  `batch` = sub-tiles of shared keys over tokens.  General form: by items up to one set of columns.
__device__ __forceinline__ bool by_items(const PlanRule &rule, long long batch, int tokens, int chunk) {
    const int sets = (tokens + rule.tg_few - 1) / rule.tg_few;
    return rule.tiles ? sets <= 1 : batch * rule.n_kv < 13000 * rule.tg_few || 17ll * sets * chunk < 10000 + 15 * chunk;
}

// x / d by magic = ceil(2^32 / d), for d of at most 256 (0 for d = 1): exact below 2^24, and a division beyond.
__device__ __forceinline__ int quotient(int x, int d, unsigned magic) { return magic && x < 1 << 24 ? (int)__umulhi((unsigned)x, magic) : x / d; }

constexpr int kAhead = 4;                       // words behind a round at most: rows that go on with its last one's run or sequence, as many as a query block has
constexpr int kFewWaves = 4;
// One workgroup, a thread per row and round of WAVES * 64 rows.  Four waves, one to a SIMD, where there are few rows: an instruction that sixteen go through
// takes four times as long; those rows are one round, so nothing of them lies before or behind it.
template <bool SHARE, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void attn_shared_plan_kernel(const int32_t *__restrict__ seq_of_token, const int32_t *__restrict__ pos_of_token, int rows,
                                                                AttnPrefix prefix, AttnShape sh, PlanRule rule, SharedPlan w) {
    constexpr int ROUND = WAVES * 64;
    constexpr bool ONE = WAVES == kFewWaves;                         // rows <= ROUND
    static_assert(WAVES >= kAhead, "a wave per word of rows ahead");
    // per sequence: its lead (-1: none), pages, whether items serve its shared keys (the sign) and their chunks; per lead: who shares
    __shared__ int lead_of[SHARE ? kShareSeqs : 1], pages_of[SHARE ? kShareSeqs : 1], rule_of[SHARE && WAVES != kFewWaves ? kShareSeqs : 1], members[SHARE ? kShareSeqs : 1];
    // per sequence, where there are enough rows for a long prompt (prompt_chunk_positions, whose rule it is): its rows of the batch, and the first one's own
    // position.  Its blocks of own keys have longer chunks: 4096 tokens alone 259 -> 230 us, behind 2000 positions of their own 425 -> 380, 6000 751 -> 598, 4096
    // beside 64 decodes 402 -> 370; 5387 rows of 242 sequences 202 -> 203.5.
    constexpr bool RUNS = SHARE && WAVES != kFewWaves;
    __shared__ int run_start[RUNS ? kShareSeqs : 1], run_end[RUNS ? kShareSeqs : 1], run_pos[RUNS ? kShareSeqs : 1];
    const bool long_prompts = RUNS && !rule.tiles && prefix.rows > kLongRun && prefix.n_seqs <= kShareSeqs;
    __shared__ int batch[2], cost[2];                                // sub-tiles of shared and of own keys; what the lists take, in 1/16 us
    __shared__ int edge_lead[WAVES + 1], edge_keys[WAVES + 1], edge_seq[WAVES + 1], edge_shift[WAVES + 1];       // the last row of each wave's 64, and of the round before
    __shared__ unsigned long long p_goes_on[WAVES + kAhead], s_goes_on[WAVES + kAhead];      // rows like the one before them: the same prefix, the same sequence
    __shared__ int sums[3][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ps = sh.page_size, max_pages = sh.max_pages_per_seq;
    const bool any = SHARE && prefix.lead != nullptr;
    // a row whose sequence or position lies outside the table attends nothing, as one of position -1
    auto inside = [&](int seq, int pos) { return (unsigned)seq < (unsigned)prefix.n_seqs && pos < max_pages * ps ? pos : -1; };
    int next_seq = -1, next_pos = -1;                                // the next round's row, on its way
    if (tid < rows) { next_seq = seq_of_token[tid]; next_pos = pos_of_token[tid]; }
    if (tid < 2) batch[tid] = cost[tid] = 0;
    if (tid <= WAVES) edge_lead[tid] = edge_keys[tid] = edge_seq[tid] = edge_shift[tid] = -1;
    if (any) {
        for (int s = tid; s < prefix.n_seqs; s += ROUND) {
            const int lead = prefix.lead[s], pages = prefix.pages[s];
            const bool ok = lead >= 0 && lead < prefix.n_seqs && pages >= 1 && pages < max_pages;
            lead_of[s] = ok ? lead : -1;
            pages_of[s] = pages;
            members[s] = 0;
        }
        __syncthreads();
        for (int s = tid; s < prefix.n_seqs; s += ROUND)
            if (lead_of[s] >= 0) atomicAdd(&members[lead_of[s]], 1);
        __syncthreads();
        // from here on: the batch's tokens behind a prefix that two sequences and more name; -1: nobody shares with this lead
        for (int s = tid; s < prefix.n_seqs; s += ROUND) members[s] = members[s] > 1 ? 0 : -1;
    }
    __syncthreads();
    struct Row { int seq, pos, lead, pages, keys; };                 // lead -1: shares nothing
    auto row_of = [&](int seq, int pos) {
        Row r{seq, pos, -1, 0, 0};
        if (any && pos >= 0 && seq >= 0 && seq < prefix.n_seqs && lead_of[seq] >= 0 && members[lead_of[seq]] >= 0 && pos >= pages_of[seq] * ps) {
            r.lead = lead_of[seq];
            r.pages = pages_of[seq];
            r.keys = r.pages * ps;
        }
        return r;
    };
    if constexpr (SHARE) {                                           // all rows of the batch, whichever of them are served here
        int shared = 0, own = 0;
        for (int t = tid; t < prefix.rows; t += ROUND) {
            const int seq = prefix.seq_of_token[t], before = prefix.seq_of_token[max(t - 1, 0)];
            const Row r = row_of(seq, inside(seq, prefix.pos_of_token[t]));
            if (r.lead >= 0) {
                atomicAdd(&members[r.lead], 1);
                shared += r.keys >> 4;
            }
            if (long_prompts) {
                if ((t == 0 || before != seq) && (unsigned)seq < (unsigned)prefix.n_seqs) { run_start[seq] = t; run_pos[seq] = r.pos - r.keys; }
                if (t > 0 && before != seq && (unsigned)before < (unsigned)prefix.n_seqs) run_end[before] = t;
                if (t + 1 == prefix.rows && (unsigned)seq < (unsigned)prefix.n_seqs) run_end[seq] = t + 1;
            }
            if (t == 0 || before != seq || (rule.tiles && (r.pos - r.keys) % rule.tg_many == 0)) own += (r.pos - r.keys + 16) >> 4;
        }
        shared = sum_all(shared);
        own = sum_all(own);
        if (lane == 0) {
            if (shared) atomicAdd(&batch[0], shared);
            if (own) atomicAdd(&batch[1], own);
        }
        __syncthreads();
    }
    const long long batch_shared = batch[0] / rule.tg_many, batch_own = batch[1];
    auto prefix_rule = [&](int lead, int keys) {
        const int ct = block_positions(rule, batch_shared, batch_own, keys);
        return by_items(rule, batch[0], members[lead], ct) ? item_positions(rule, batch_own, 2 * keys) | (int)0x80000000u : ct;
    };
    if (any && !ONE) {                                               // (one round: every row for itself, and no barrier)
        for (int s = tid; s < prefix.n_seqs; s += ROUND) {
            const int lead = lead_of[s];
            if (lead >= 0 && members[lead] >= 0) rule_of[s] = prefix_rule(lead, pages_of[s] * ps);
        }
        __syncthreads();
    }
    // a value per wave, joined: over the waves below this one, and over all
    struct Joined { int below, all; };
    auto over_waves = [&](const int *row, int empty, auto op) {
        if constexpr (ONE) {
            Joined j{empty, empty};
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                if (k < wave) j.below = op(j.below, row[k]);
                j.all = op(j.all, row[k]);
            }
            return j;
        }
        const int x = scan_wave(lane < WAVES ? row[lane] : empty, empty, op), at = __builtin_amdgcn_readfirstlane(wave);
        return Joined{at ? __builtin_amdgcn_readlane(x, at - 1) : empty, __builtin_amdgcn_readlane(x, 63)};
    };
    // The run that this thread's row lies in, of rows that each go on like the one before (a bit each; mine: this wave's): its first row, and how many of it are
    // behind this row, up to rule.ahead words past the round.  before: the first row of the run that the round's last row lies in.
    struct Run { int start, behind; };
    auto run_of = [&](const unsigned long long *words, unsigned long long mine, int t0, int &before) {
        const int at = __builtin_amdgcn_readfirstlane(wave);
        const unsigned long long x = lane < (ONE ? WAVES : WAVES + rule.ahead) ? words[lane] : 0ull;
        const int ones = x == ~0ull ? 64 : __ffsll(~x) - 1, last = 63 - __clzll((long long)~x);         // rows in front that go on, the last that does not
        const unsigned long long cut = __ballot(x != ~0ull), below = cut & ((1ull << at) - 1), all = cut & ((1ull << WAVES) - 1);
        const int next = __ffsll(cut >> (at + 1)) + at, beyond = (next - at - 1) * 64 + __builtin_amdgcn_readlane(ones, next);
        auto start_in = [&](unsigned long long words_cut) {
            const int k = __builtin_amdgcn_readfirstlane(63 - __clzll((long long)words_cut));
            return t0 + k * 64 + __builtin_amdgcn_readlane(last, k);
        };
        const unsigned long long own = ~mine & ((2ull << lane) - 1), rest = ~(lane == 63 ? 0ull : mine >> (lane + 1));
        const int start = below ? start_in(below) : before, run = __ffsll(rest) - 1;
        if (all) before = start_in(all);
        return Run{own ? t0 + at * 64 + 63 - __clzll((long long)own) : start, run < 63 - lane ? run : 63 - lane + beyond};
    };
    int run_before = -1, seq_before_run = -1, before[3] = {0, 0, 0}; // the last run's and sequence's first rows; entries of items, p_blocks, s_blocks so far
    int cost_items = 0, cost_blocks = 0;
    for (int t0 = 0; t0 < rows; t0 += ROUND) {
        const int t = t0 + tid;
        const Row r = row_of(next_seq, inside(next_seq, next_pos));
        const bool on = r.lead >= 0, live = t < rows;
        const int s_seq = !live ? -2 : r.pos < 0 ? -3 - t : r.seq * max_pages + r.pages, p = r.pos - r.keys;
        const int shift = p - t;                                     // the same where positions follow one another, as items and query blocks take them to
        // rows behind this round that go on with its last one's run or sequence
        int ahead_seq = -1, ahead_pos = -1;
        if (!ONE && wave < rule.ahead && t0 + ROUND + tid < rows) { ahead_seq = seq_of_token[t0 + ROUND + tid]; ahead_pos = pos_of_token[t0 + ROUND + tid]; }
        next_seq = next_pos = -1;
        if (!ONE && t + ROUND < rows) { next_seq = seq_of_token[t + ROUND]; next_pos = pos_of_token[t + ROUND]; }
        if (lane == 63) { edge_lead[wave + 1] = on ? r.lead : -1; edge_keys[wave + 1] = r.keys; edge_seq[wave + 1] = s_seq; edge_shift[wave + 1] = shift; }
        __syncthreads();
        int lead_before = __shfl_up(on ? r.lead : -1, 1, 64), keys_before = __shfl_up(r.keys, 1, 64), seq_before = __shfl_up(s_seq, 1, 64), shift_before = __shfl_up(shift, 1, 64);
        if (lane == 0) { lead_before = edge_lead[wave]; keys_before = edge_keys[wave]; seq_before = edge_seq[wave]; shift_before = edge_shift[wave]; }
        const bool same_prefix = on && lead_before == r.lead && keys_before == r.keys, same_seq = live && seq_before == s_seq && shift_before == shift;
        const unsigned long long p_mask = __ballot(same_prefix), s_mask = __ballot(same_seq);
        if (lane == 0) { p_goes_on[wave] = p_mask; s_goes_on[wave] = s_mask; }
        if (!ONE && wave < rule.ahead) {
            const Row x = row_of(ahead_seq, inside(ahead_seq, ahead_pos));
            const unsigned long long pm = __ballot(x.lead >= 0 && x.lead == edge_lead[WAVES] && x.keys == edge_keys[WAVES]);
            const unsigned long long sm = __ballot(x.pos >= 0 && x.seq * max_pages + x.pages == edge_seq[WAVES] && x.pos - x.keys - (t0 + ROUND + tid) == edge_shift[WAVES]);
            if (lane == 0) { p_goes_on[WAVES + wave] = pm; s_goes_on[WAVES + wave] = sm; }
        }
        __syncthreads();
        const Run p_run = run_of(p_goes_on, p_mask, t0, run_before), s_run = run_of(s_goes_on, s_mask, t0, seq_before_run);
        if (!ONE && tid == 0) { edge_lead[0] = edge_lead[WAVES]; edge_keys[0] = edge_keys[WAVES]; edge_seq[0] = edge_seq[WAVES]; edge_shift[0] = edge_shift[WAVES]; }   // (read again behind the next barriers)
        int p_tok = 0, p_n = 0, p_ct = 64, s_tok = 0, s_n = 0, s_ct = 64;              // what row t leads: tokens and chunks
        bool few = false, single = false;
        if (on) {
            const int r_rule = ONE ? prefix_rule(r.lead, r.keys) : rule_of[r.seq];
            few = r_rule < 0;
            p_ct = r_rule & 0x7fffffff;
        }
        const int width = few ? rule.tg_few : rule.tg_many;
        const int p_at = t - p_run.start, s_at = t - s_run.start;
        const bool leads = on && p_at == quotient(p_at, width, few ? rule.few_magic : rule.many_magic) * width;
        if constexpr (SHARE) {
            if (leads) {
                p_tok = min(width, 1 + p_run.behind);
                p_n = (r.keys - 1 + p_ct) / p_ct;
            }
            if (live && r.pos >= 0) {
                const int tg = rule.tg_many, block = quotient(p, tg, rule.many_magic);
                single = s_at + 1 + s_run.behind <= rule.short_tokens;
                const int reach = (block + 1) * tg, prompt = long_prompts ? run_end[r.seq] - run_start[r.seq] : 0;
                s_ct = single ? item_positions(rule, batch_own, p + s_run.behind + 1) : rule.tiles ? item_positions(rule, batch_own, reach) :
                       prompt <= kLongRun ? prefill_chunk_positions(reach) : prefill_run_chunk_positions(reach, tg, rule.n_kv, prompt, run_pos[r.seq] + (prompt + 1) / 2);
                const int at = single ? s_at : same_seq ? p - block * tg : 0;
                if (at == 0) {                                                                     // rows of the sequence in this item, or in its aligned block
                    s_tok = single ? 1 + s_run.behind : min(tg - (p - block * tg), 1 + s_run.behind);
                    s_n = (p + s_tok - 1 + s_ct) / s_ct;                                          // chunks the last of them reaches
                }
            }
            // a position of an item 512 bytes at 19.5 GB/s; beside items, a query block's tile of 64 positions 2 us and up to 1 more where all its columns are live, a
            // block and chunk 20 us around its tiles
            const int p_subs = p_n ? r.keys >> 4 : 0, s_subs = s_n ? (p + s_tok + 15) >> 4 : 0;
            cost_items += 7 * ((few ? p_subs : 0) + (single ? s_subs : 0));
            auto block_cost = [&](int subs, int tok, int n) { return 8 * subs + quotient(4 * subs, rule.tg_many, rule.many_magic) * tok + n * 320; };
            if (!few && p_n) cost_blocks += block_cost(p_subs, p_tok, p_n);
            if (!single && s_n) cost_blocks += block_cost(s_subs, s_tok, s_n);
        }
        const int mine[3] = {(few ? p_n : 0) + (single ? s_n : 0), few ? 0 : p_n, single ? 0 : s_n};
        int start[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int incl = sum_up(mine[k]);
            if (lane == 63) sums[k][wave] = incl;
            start[k] = before[k] + incl - mine[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const auto [below, all] = over_waves(sums[k], 0, [](int a, int b) { return a + b; });
            start[k] += below;
            before[k] += all;
        }
        if (live) {
            w.s_seq[t] = r.pos < 0 ? -1 : s_seq;
            w.s_pos[t] = r.pos < 0 ? -1 : p;
            w.p_pos[t] = on ? r.keys - 1 : -1;
            w.p_seq[t] = on ? r.lead * max_pages : -1;
            w.p_ct[t] = p_ct;
            w.s_ct[t] = SHARE ? s_ct : rule.most_positions;
            if constexpr (SHARE) {
                int32_t *at = few ? w.items + 2 + 2 * (size_t)start[0] : w.p_blocks + 2 + 2 * (size_t)start[1];
                for (int c = 0; c < p_n; ++c) { *at++ = t; *at++ = c | (p_tok << 20); }
                at = single ? w.items + 2 + 2 * (size_t)(start[0] + (few ? p_n : 0)) : w.s_blocks + 2 + 2 * (size_t)start[2];
                for (int c = 0; c < s_n; ++c) { *at++ = single ? t | kOwnItem : t; *at++ = c | (s_tok << 20); }
            }
        }
        if (ONE) break;
        __syncthreads();
    }
    if constexpr (SHARE) {
        cost_items = sum_all(cost_items);
        cost_blocks = sum_all(cost_blocks);
        if (lane == 0) {
            if (cost_items) atomicAdd(&cost[0], cost_items);
            if (cost_blocks) atomicAdd(&cost[1], cost_blocks);
        }
        __syncthreads();
        if (tid < 2) w.cost[tid] = cost[tid] * (1.0f / 16);
        if (tid == 0) {
            w.items[0] = before[0];
            w.p_blocks[0] = before[1];
            w.s_blocks[0] = before[2];
            w.items[1] = w.p_blocks[1] = w.s_blocks[1] = 0;
        }
    }
}

}  // namespace

// The shapes that the forms of this operator take: the layer's fast ones, and larger pages.
static bool lists_shape(int dtype, const AttnShape &sh) {
    AttnShape small = sh;
    if (sh.page_size % 16 == 0) small.page_size = 16;
    return attention_mfma_supported(dtype, small);
}

int attn_prefix_max_chunks(int dtype, const AttnShape &sh) {
    const long positions = (long)sh.max_pages_per_seq * sh.page_size;
    if (!lists_shape(dtype, sh) && !attn_tile_shape(sh)) return 1;
    const long most = std::max<long>(32, (positions + 8191) / 8192);
    return (int)std::max<long>(1, std::min<long>(most, (positions + 63) / 64));
}

int attn_own_max_chunks(int dtype, const AttnShape &sh) {
    const int chunks = (sh.max_pages_per_seq + sh.chunk_pages - 1) / sh.chunk_pages;
    if (!lists_shape(dtype, sh) && !attn_tile_shape(sh)) return chunks;
    const long positions = (long)sh.max_pages_per_seq * sh.page_size;
    const int items = std::max(chunks, (int)std::min<long>(64, (positions + 63) / 64));
    return lists_shape(dtype, sh) ? std::max(items, attn_prefill_max_chunks(positions)) : items;
}

size_t attn_shared_plan_words(const AttnShape &sh, const AttnPrefix &prefix, int rows) {
    const size_t own = (size_t)sh.max_chunks * rows, shared = (size_t)prefix.max_chunks * rows;
    return (size_t)rows * 6 + 8 + 4 * (own + shared);          // (for rows together no more than for each of them alone)
}

SharedPlan attn_shared_plan(int32_t *plan, const AttnShape &sh, const AttnPrefix &prefix, int rows) {
    SharedPlan w;
    int32_t *at = plan;
    for (int32_t **a : {&w.p_seq, &w.p_pos, &w.p_ct, &w.s_seq, &w.s_pos, &w.s_ct}) { *a = at; at += rows; }
    const size_t own = (size_t)sh.max_chunks * rows, shared = (size_t)prefix.max_chunks * rows;
    w.cost = (float *)at;
    w.items = at + 2;
    w.p_blocks = w.items + 2 + 2 * (own + shared);
    w.s_blocks = w.p_blocks + 2 + 2 * shared;
    return w;
}

AttnForm attn_shared_form(int dtype, const AttnShape &sh, const void *k_cache, const void *v_cache) {
    return lists_shape(dtype, sh) && !(((uintptr_t)k_cache | (uintptr_t)v_cache) & 15) ? SHARE_LISTS : attn_tile_takes(sh, k_cache, v_cache) ? SHARE_TILES : SHARE_NOTHING;
}

hipError_t launch_attn_shared_plan(AttnForm form, const int32_t *seq_of_token, const int32_t *pos_of_token, const AttnShape &sh, const AttnPrefix &prefix, int rows,
                                   const SharedPlan &w, hipStream_t s) {
    const int G = sh.n_q / sh.n_kv, TG = G <= 16 ? 16 / G : 1;
    AttnPrefix p = prefix;
    if (p.n_seqs > kShareSeqs) p.lead = nullptr;
    const int many = form == SHARE_LISTS ? attn_prefill_block_tokens(sh) : 4 * TG;
    auto magic = [](int d) { return (unsigned)((0x100000000ull + d - 1) / d); };
    const PlanRule rule{many, TG, magic(many), magic(TG), (many + 63) / 64, form == SHARE_LISTS ? TG : 1, sh.chunk_pages * sh.page_size, form == SHARE_TILES ? 128 : 64,
                        form == SHARE_TILES || sh.page_size == 16 ? 128 : 64, sh.n_kv, form == SHARE_TILES};
    const bool small = std::max(rows, prefix.rows) <= kFewWaves * 64 && prefix.n_seqs <= 1024;       // (340 rows: 54 us in one round of 16 waves, 57 in two of 4)
    const auto kernel = form == SHARE_NOTHING ? attn_shared_plan_kernel<false, 16> : small ? attn_shared_plan_kernel<true, kFewWaves> : attn_shared_plan_kernel<true, 16>;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(form != SHARE_NOTHING && small ? kFewWaves * 64 : 1024), 0, s, seq_of_token, pos_of_token, rows, p, sh, rule, w);
    return hipGetLastError();
}

}  // namespace dyn

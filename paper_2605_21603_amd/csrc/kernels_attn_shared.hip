// Attention of a batch whose sequences share prefixes: the shared pages are read once for all that share them.
//
// A token at position p attends keys 0 .. p of its sequence.  Softmax over two sets of keys is that of each, merged:
//     m = max(m1, m2),  o = (e^(m1 - m) o1 + e^(m2 - m) o2) / (e^(m1 - m) l1 + e^(m2 - m) l2)
// with o_i, l_i the sums of e^(s - m_i) v and e^(s - m_i) over set i.  So the first P keys, which many sequences have in common, become
// one attention of all their tokens against the same pages - a product with many columns, as a prompt's - and the keys behind
// them an attention of every sequence for itself, as a decode's or a prompt's that starts at P.  Three launches: the plan
// (kernels_attn_shared_plan.hip), the keys (attn_shared_kernel, or attn_tile of kernels_attn_generic.hip for what it does not
// take), and the merge of a row's chunks.
// 32 q heads, 8 kv heads, 128 wide, caches out of reach of the last call, plan + keys + merge: 5 tokens behind 512 positions 5.2 + 7.3 + 4.0 us; 64 behind 2048 with
// 16 to 1024 of their own, 162 MB, 5.9 + 49 + 5.2; 256 on 4 prefixes, 1.19 GB, 6.6 + 252 (4.7 TB/s) + 9.5; 12 prompts of 33 to 300 tokens behind 4096 positions, 1.08e11
// operations, 13 + 132 (0.82 PFLOP/s) + 14.
// A token's product has columns of tokens that do not see it, where its probability is zero: infinities and NaN among its values are taken out of the product
// and put back for the columns that see them, so that for the others it is as any finite value (64 sequences of 4 tokens, one of them with NaN: 65.6 -> 66.8 us).
#include <algorithm>
#include <atomic>

#include "attn_prefill.h"
#include "attn_shared_plan.h"
#include "common.h"

namespace dyn {

namespace {

constexpr int HD = 128, TILE = 2;         // head dim; sub-tiles of 16 positions to a register buffer

struct SharedArgs {
    const bf16_t *q, *k, *v;
    const int32_t *block_table;
    SharedPlan plan;
    AttnShape sh;                         // rows of a table of one wide row; max_chunks: of both halves
    int ld_q, shared_slots;               // partials of own keys lie behind shared_slots chunks of shared ones
    float *part_o, *part_ml;
    prefill::SubTiles page;
};

// One wave's work: up to 16 columns (a token and a q head each) against one chunk of one kv head.  Shared keys all of them see; of own keys, each token
// one more than the one before it.
struct Item {
    int t, n_tok, own, c, g;              // first token row, tokens, whose keys, chunk, kv head
    int first, last, end;                 // the chunk's sub-tiles; the first position past it
    int full;                             // the first position that its first token does not see
    const int32_t *table;
};

__device__ __forceinline__ Item fetch_item(const SharedArgs &a, int i) {
    Item m;
    const int e = i / a.sh.n_kv, row = a.plan.items[2 + 2 * e], packed = a.plan.items[3 + 2 * e];
    m.g = i - e * a.sh.n_kv;
    m.t = row & (kOwnItem - 1);
    m.own = row >> 30;
    m.c = packed & 0xfffff;
    m.n_tok = packed >> 20;
    const int keys = (m.own ? a.plan.s_pos : a.plan.p_pos)[m.t] + (m.own ? m.n_tok : 1);
    m.table = a.block_table + (m.own ? a.plan.s_seq : a.plan.p_seq)[m.t];
    // chunks of equal size up to rounding, a function of the half's own length; fixed ones where tokens of different lengths share them
    const int subs = (keys + 15) >> 4, most = (m.own ? a.plan.s_ct : a.plan.p_ct)[m.t] >> 4, n = (subs + most - 1) / most;
    const int per = m.own && m.n_tok > 1 ? most : (subs + n - 1) / n;
    m.first = m.c * per;
    m.last = min(m.first + per, subs) - 1;
    m.end = min(keys, (m.last + 1) * 16);
    m.full = m.own ? min(m.end, keys - m.n_tok + 1) : m.end;
    return m;
}

// The items: every n_blocks-th from `block` on is this workgroup's, and its waves take them as they come, from a counter in LDS.  (A fixed share
// to every wave: of the two waves of a SIMD the older gets its loads first, and with equal shares - 256 tokens of 1024 keys - the older ones were through
// after 149 us and the others after 196.)  K and V go from memory straight into MFMA operand layout,
//     S[16 pos, 16 cols]  = K_sub[16, 128] Q^T[128, 16]       (4 x mfma 16x16x32 per sub-tile)
//     O^T[128, 16 cols]  += V^T[128, 32] P[32, 16]            (8 x mfma 16x16x32 per pair of sub-tiles and part of P)
// with the D layout of the first product (lane: column l % 16, positions 4 (l / 16) + r) the B layout of the second.  Two register
// buffers of 32 positions; the last pair of a chunk is followed by the first of the wave's next item, whose indices were
// fetched while this one was multiplied.
template <bool WIDE_PAGES>
__device__ __forceinline__ void serve_items(const SharedArgs &a, int block, int n_blocks, int *taken) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
    const AttnShape &sh = a.sh;
    const int n_items = a.plan.items[0] * sh.n_kv;
    const int G = sh.n_q / sh.n_kv, col_tok = lr / G, col_head = lr - col_tok * G;
    const float scale = 1.4426950408889634f / sqrtf((float)HD);        // log2(e) / sqrt(d)
    auto take = [&]() {
        int k = 0;
        if (lane == 0) k = atomicAdd(taken, 1);
        return block + __builtin_amdgcn_readfirstlane(k) * n_blocks;
    };
    int item = take();
    if (item >= n_items) return;

    auto fetch = [&](int i) { return fetch_item(a, i); };
    u32x4 kr[2][TILE][4];
    u32x2 vr[2][TILE][8];
    bf16x8 q[4], q_next[4];
    auto load = [&](auto buf, const Item &m, int tile) {
        constexpr int B = decltype(buf)::value;
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            const int sub = min(m.first + tile * TILE + i, m.last), per = WIDE_PAGES ? a.page.per : 1, at = WIDE_PAGES ? a.page.page_of(sub) : sub, slot = (sub - at * per) * 16, ps = 16 * per;
            const size_t page = (size_t)m.table[at] * sh.n_kv + m.g;
            const bf16_t *kp = a.k + (page * ps + slot + lr) * HD + 8 * lq, *vp = a.v + (page * HD + lr) * ps + slot + 4 * lq;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) kr[B][i][ks] = *reinterpret_cast<const u32x4 *>(kp + ks * 32);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) vr[B][i][dt] = *reinterpret_cast<const u32x2 *>(vp + dt * 16 * ps);
        }
    };
    auto load_q = [&](bf16x8 (&dst)[4], const Item &m) {
        const bool live = col_tok < m.n_tok;
        const bf16_t *qp = a.q + (size_t)(m.t + (live ? col_tok : 0)) * a.ld_q + (m.g * G + col_head) * HD + 8 * lq;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            u32x4 x = *reinterpret_cast<const u32x4 *>(qp + ks * 32);
            if (!live) x = u32x4{0u, 0u, 0u, 0u};
            dst[ks] = __builtin_bit_cast(bf16x8, x);
        }
    };
    f32x4 acc[8];
    float m_run, l_run;
    bool odd;                                // of the chunk: infinities or NaN were taken out
    auto multiply = [&](auto buf, const Item &m, int tile) {
        constexpr int B = decltype(buf)::value;
        const int at = (m.first + tile * TILE) * 16;
        f32x4 s[TILE];
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kr[B][i][ks]), q[ks], s[i], 0, 0, 0);
            s[i] *= scale;
        }
        // the chunk ends in this tile, or some token does not see all of it (wave-uniform)
        if (at + 16 * TILE > m.full) {
            const int seen = min(m.end, m.full + col_tok);               // by this lane's column
#pragma unroll
            for (int i = 0; i < TILE; ++i) {
                const int n = m.end - (at + 16 * i + 4 * lq);            // valid positions of this lane's four
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at + 16 * i + 4 * lq + r >= seen) s[i][r] = -INFINITY;
                // what lies past them must not meet its zero probability (0 * NaN)
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    vr[B][i][dt][0] &= (n > 0 ? 0x0000ffffu : 0u) | (n > 1 ? 0xffff0000u : 0u);
                    vr[B][i][dt][1] &= (n > 2 ? 0x0000ffffu : 0u) | (n > 3 ? 0xffff0000u : 0u);
                }
                // of a token that only later columns see, infinities and NaN neither: they come back behind the chunk for the columns that see them
                if (m.full < m.end) {
                    bool found = false;
#pragma unroll
                    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t keep = prefill::late_mask(vr[B][i][dt][h], at + 16 * i + 4 * lq + 2 * h, m.full);
                            vr[B][i][dt][h] &= keep;
                            found |= keep != ~0u;
                        }
                    odd |= __any(found) != 0;
                }
            }
        }
        float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
        for (int i = 1; i < TILE; ++i) mx = fmaxf(mx, fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3])));
        mx = prefill::quad_max(mx);
        const float m_new = fmaxf(m_run, mx), ref = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m_run - ref);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] *= alpha;
        // probabilities go into the matrix product in NP bf16 parts (parts_of_p), and what goes in is what is summed
        constexpr int NP = prefill::parts_of_p(WIDE_PAGES);
        u32x2 w[TILE][NP];
#pragma unroll
        for (int i = 0; i < TILE; ++i) {
            f32x4 p;
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[i][r] - ref);
            prefill::bf16_parts<NP>(p, w[i]);
#pragma unroll
            for (int k = NP - 1; k >= 0; --k)
                l_run += (__uint_as_float(w[i][k][0] << 16) + __uint_as_float(w[i][k][0] & 0xffff0000u)) + (__uint_as_float(w[i][k][1] << 16) + __uint_as_float(w[i][k][1] & 0xffff0000u));
        }
#pragma unroll
        for (int i = 0; i < TILE; i += 2) {
#pragma unroll
            for (int k = NP - 1; k >= 0; --k) {
                const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{w[i][k][0], w[i][k][1], w[i + 1][k][0], w[i + 1][k][1]});
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const u32x2 x = vr[B][i][dt], y = vr[B][i + 1][dt];
                    acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{x[0], x[1], y[0], y[1]}), pb, acc[dt], 0, 0, 0);
                }
            }
        }
    };
    const std::integral_constant<int, 0> b0;
    const std::integral_constant<int, 1> b1;
    Item cur = fetch(item);
    load_q(q, cur);
    load(b0, cur, 0);
    while (true) {
        const int next = take();
        const bool more = next < n_items;
        const Item nxt = fetch(more ? next : item);       // the last one "prefetches" itself: harmless loads, no branch
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run = -INFINITY;
        l_run = 0.f;
        odd = false;
        const int pairs = (cur.last - cur.first + 2 * TILE) / (2 * TILE);     // an odd tile at the end is walked masked
        for (int pr = 0; pr < pairs; ++pr) {
            load(b1, cur, 2 * pr + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(b0, cur, 2 * pr);
            __builtin_amdgcn_sched_barrier(0);
            const bool last = pr + 1 == pairs;
            load_q(q_next, nxt);
            load(b0, last ? nxt : cur, last ? 0 : 2 * pr + 2);
            __builtin_amdgcn_sched_barrier(0);
            multiply(b1, cur, 2 * pr + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (odd) {
#pragma clang loop unroll(disable)
            for (int at = max(cur.full, cur.first * 16); at < cur.end; ++at) {
                const int sub = at >> 4, per = WIDE_PAGES ? a.page.per : 1, in = WIDE_PAGES ? a.page.page_of(sub) : sub, ps = 16 * per;
                const bf16_t *vp = a.v + (((size_t)cur.table[in] * sh.n_kv + cur.g) * HD + 4 * lq) * ps + at - in * ps;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float x = prefill::odd_or_0(vp[(dt * 16 + r) * ps]);
                        acc[dt][r] += at < cur.full + col_tok ? x : 0.f;
                    }
            }
        }
        float l = l_run;
        l += __shfl_xor(l, 16, 64);
        l += __shfl_xor(l, 32, 64);
        if (col_tok < cur.n_tok && cur.full + col_tok > cur.first * 16) {    // (a token that ends before the chunk has no partial of it)
            const size_t at = part_index(sh, cur.t + col_tok, cur.g * G + col_head, cur.own ? a.shared_slots + cur.c : cur.c);
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4 *>(a.part_o + at * HD + dt * 16 + 4 * lq) = acc[dt];
            if (lq == 0) {
                a.part_ml[at * 2] = m_run;
                a.part_ml[at * 2 + 1] = l;
            }
        }
        if (!more) break;
        item = next;
        cur = nxt;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) q[ks] = q_next[ks];
    }
}

// All keys of a dispatch in one launch, a workgroup of eight waves per CU: the first claim query blocks (of shared keys, then of own
// ones), the others serve the items of both and then claim query blocks too.  Items wait for memory and query blocks for the matrix
// cores (attn_mixed_kernel, kernels_attn_mfma.hip).  Items for the first workgroups too, behind their query blocks, cost registers: 64 tokens behind 2048 positions
// 64.5 -> 67.7 us.
template <bool WIDE_PAGES>
__global__ __launch_bounds__(prefill::kWaves * 64, 1) void attn_shared_kernel(SharedArgs a) {
    const SharedPlan &w = a.plan;
    __shared__ int taken;
    if (threadIdx.x == 0) taken = 0;
    __syncthreads();
    const int groups = gridDim.x, n_blocks = w.p_blocks[0] + w.s_blocks[0];
    const int first = n_blocks == 0 ? 0 : w.items[0] == 0 ? groups : mixed_share(n_blocks * a.sh.n_kv, w.cost[1], w.cost[0], groups);
    if ((int)blockIdx.x >= first) serve_items<WIDE_PAGES>(a, (int)blockIdx.x - first, groups - first, &taken);
    const size_t behind = part_index(a.sh, 0, 0, a.shared_slots);
#pragma clang loop unroll(disable)
    for (int own = 0; own < 2; ++own) {
        int32_t *const list = own ? w.s_blocks : w.p_blocks;
        if (list[0] == 0) continue;
        prefill::attn_prefill_items<true, WIDE_PAGES>(a.q, own ? w.s_seq : w.p_seq, own ? w.s_pos : w.p_pos, a.block_table, a.k, a.v, nullptr, 0,
                                          a.part_o + (own ? behind * HD : 0), a.part_ml + (own ? behind * 2 : 0), a.sh, list, list + 1, own ? w.s_ct : w.p_ct, a.ld_q, a.page);
    }
}

// Merge of a row's partials, shared chunks first, in order; four head-dim indices to a lane, two sets of them in the WIDE form (head dims above
// 128).  Where there are rows to fill the chip a half-wave merges a (token, q head); else (SPLIT) a workgroup does, its eight half-waves every
// eighth chunk each and the eight results in order through LDS.  A row without keys is zero.  What it costs is two dependent loads, of the row's chunk counts and
// of its partials, so the first of those are all on their way beside the maxima and sums that weigh them.
template <typename T, bool BASE2, bool WIDE, bool SPLIT>
__global__ __launch_bounds__(256, SPLIT ? 1 : WIDE ? 6 : 8) void attn_shared_combine_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                                  const int32_t *__restrict__ p_pos, const int32_t *__restrict__ p_ct,
                                                                  const int32_t *__restrict__ s_pos, const int32_t *__restrict__ s_ct,
                                                                  int shared_slots, T *__restrict__ out, int ld_out, AttnShape sh,
                                                                  int32_t *__restrict__ counter0, int32_t *__restrict__ counter1) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    constexpr int SETS = WIDE ? 2 : 1, MOST_LOADS = 8 / SETS, STEP = SPLIT ? 8 : 1;
    // the lists' query blocks have all been claimed: from the start again for the next layer
    if (counter0 && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 2) *(threadIdx.x ? counter1 : counter0) = 0;
    const int t = blockIdx.x, sub = threadIdx.x & 31, half = threadIdx.x >> 5, d = sh.head_dim, h = SPLIT ? (int)blockIdx.y : (int)blockIdx.y * 8 + half;
    if (h >= sh.n_q) return;
    const int pp = p_pos[t], sp = s_pos[t], pc = p_ct[t], sc = s_ct[t];
    const int n_shared = pp < 0 ? 0 : (pp + pc) / pc, n = n_shared + (sp < 0 ? 0 : (sp + sc) / sc);
    const int c0 = SPLIT ? half : 0, count = (n - c0 + STEP - 1) / STEP;                     // chunks c0, c0 + STEP, ...
    f32x4 acc[SETS];
#pragma unroll
    for (int k = 0; k < SETS; ++k) acc[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    float M = -INFINITY, L = 0.f;
    auto weight = [](float x) { return BASE2 ? exp2f(x) : expf(x); };
    if (count > 0) {
        const size_t first = part_index(sh, t, h, 0), next = sh.n_q;                         // from a chunk to the one behind it
        auto at = [&](int i) {
            const int c = c0 + i * STEP;
            return first + (size_t)(c < n_shared ? c : shared_slots + c - n_shared) * next;
        };
        auto ml_of = [&](int i) { return i < count ? *reinterpret_cast<const f32x2 *>(part_ml + at(i) * 2) : f32x2{-INFINITY, 0.f}; };
        auto walk = [&](auto loads) {
            constexpr int LOADS = decltype(loads)::value;
            f32x4 v[LOADS][SETS];
            auto load = [&](int i0) {
#pragma unroll
                for (int j = 0; j < LOADS; ++j)
#pragma unroll
                    for (int k = 0; k < SETS; ++k) v[j][k] = *reinterpret_cast<const f32x4 *>(part_o + at(min(i0 + j, count - 1)) * d + min(sub * 4 + k * 128, d - 4));
            };
            f32x2 ml = ml_of(sub);
            load(0);
            M = ml[0];
            for (int i = sub + 32; i < count; i += 32) M = fmaxf(M, ml_of(i)[0]);
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 32));
            for (int i0 = 0; i0 < count; i0 += 32) {
                if (i0) ml = ml_of(i0 + sub);
                const float wgt = weight(ml[0] - M);                                              // 0 past the last chunk
                L += wgt * ml[1];
                for (int j0 = 0; j0 < 32 && i0 + j0 < count; j0 += LOADS) {
                    if (i0 + j0) load(i0 + j0);
#pragma unroll
                    for (int j = 0; j < LOADS; ++j) {
                        {
                            const float wj = __shfl(wgt, j0 + j, 32);
#pragma unroll
                            for (int k = 0; k < SETS; ++k) acc[k] += v[j][k] * wj;
                        }
                    }
                }
            }
        };
        // (rows of two to four chunks, prompts': 16 loads each, most of them the last chunk's again, took 24 us for 1563 rows of 32 heads, 4 take 19; and with 8 for
        // more chunks all registers of eight waves to a SIMD do: 5387 rows 75, 64 and so 45 us)
        if (!SPLIT && n <= 4) walk(std::integral_constant<int, 4>());
        else walk(std::integral_constant<int, MOST_LOADS>());
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) L += __shfl_xor(L, off, 32);
    }
    if constexpr (SPLIT) {
        __shared__ f32x4 split_o[8][32 * SETS];
        __shared__ float split_ml[8][2];
#pragma unroll
        for (int k = 0; k < SETS; ++k) split_o[half][sub + 32 * k] = acc[k];
        if (sub == 0) { split_ml[half][0] = M; split_ml[half][1] = L; }
        __syncthreads();
        if (half) return;
#pragma unroll
        for (int j = 1; j < 8; ++j) M = fmaxf(M, split_ml[j][0]);
        if (n) {
            const float w0 = weight(split_ml[0][0] - M);
            L *= w0;
#pragma unroll
            for (int k = 0; k < SETS; ++k) acc[k] *= w0;
#pragma unroll
            for (int j = 1; j < 8; ++j) {
                const float w = weight(split_ml[j][0] - M);                                   // 0 of a half-wave without a chunk
                L += w * split_ml[j][1];
#pragma unroll
                for (int k = 0; k < SETS; ++k) acc[k] += split_o[j][sub + 32 * k] * w;
            }
        }
    }
    const float inv = n ? 1.0f / L : 0.f;
    T *const y = out + (size_t)t * ld_out + h * d;
#pragma unroll
    for (int k = 0; k < SETS; ++k) {
        const int i = sub * 4 + k * 128;
        if (i < d) {
            if constexpr (sizeof(T) == 2) {
                u32x2 w;
                w[0] = (uint32_t)f2bf(acc[k][0] * inv) | ((uint32_t)f2bf(acc[k][1] * inv) << 16);
                w[1] = (uint32_t)f2bf(acc[k][2] * inv) | ((uint32_t)f2bf(acc[k][3] * inv) << 16);
                *reinterpret_cast<u32x2 *>(y + i) = w;
            } else {
                *reinterpret_cast<f32x4 *>(y + i) = acc[k] * inv;
            }
        }
    }
}

}  // namespace

hipError_t launch_attention_shared(int dtype, const void *q, int ld_q, const int32_t *seq_of_token, const int32_t *pos_of_token, const int32_t *block_table,
                                   const void *k_cache, const void *v_cache, void *out, int ld_out, float *part_o, float *part_ml, int32_t *plan,
                                   const AttnShape &sh, const AttnPrefix &prefix, int rows, hipStream_t s, hipEvent_t mid, hipEvent_t pre, int layer) {
    if (rows <= 0) return hipSuccess;
    if (rows >= 1 << 24) return hipErrorInvalidConfiguration;
    const AttnForm form = attn_shared_form(dtype, sh, k_cache, v_cache);
    const SharedPlan w = attn_shared_plan(plan, sh, prefix, rows);
    hipError_t e = layer > 0 ? hipSuccess : launch_attn_shared_plan(form, seq_of_token, pos_of_token, sh, prefix, rows, w, s);
    if (e == hipSuccess && pre) e = hipEventRecord(pre, s);
    if (e != hipSuccess) return e;
    AttnShape part = sh;
    part.max_pages_per_seq = 1;                     // the halves' arrays hold offsets into the table
    part.max_chunks = sh.max_chunks + prefix.max_chunks;
    if (form == SHARE_LISTS) {
        const auto kernel = sh.page_size == 16 ? attn_shared_kernel<false> : attn_shared_kernel<true>;
        static std::atomic<unsigned long long> attr_set[2];               // a bit per device
        int device = 0;
        if ((e = hipGetDevice(&device)) != hipSuccess) return e;
        const unsigned long long bit = 1ull << (device & 63);
        if (!(attr_set[sh.page_size != 16] & bit)) {
            e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, prefill::lds_bytes());
            if (e != hipSuccess) return e;
            attr_set[sh.page_size != 16] |= bit;
        }
        const SharedArgs a{(const bf16_t *)q, (const bf16_t *)k_cache, (const bf16_t *)v_cache, block_table, w, part, ld_q, prefix.max_chunks, part_o,
                           part_ml, prefill::SubTiles{sh.page_size / 16, (unsigned)((0x100000000ull + sh.page_size / 16 - 1) / (sh.page_size / 16))}};
        const long most = (long)rows * sh.n_kv * part.max_chunks;
        const int cus = sh.n_cus > 0 && sh.n_cus < 256 ? sh.n_cus : 256;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<long>(most, cus)), dim3(prefill::kWaves * 64), prefill::lds_bytes(), s, a);
        e = hipGetLastError();
    } else if (form == SHARE_TILES) {
        e = launch_attention_parts(dtype, q, ld_q, block_table, k_cache, v_cache, part_o, part_ml, part, w, prefix.max_chunks, rows, s);
    } else {
        const size_t behind = part_index(part, 0, 0, prefix.max_chunks);
        e = launch_attention_own(dtype, q, ld_q, w.s_seq, w.s_pos, block_table, k_cache, v_cache, part_o + behind * sh.head_dim, part_ml + behind * 2, part, rows, s);
    }
    if (e == hipSuccess && mid) e = hipEventRecord(mid, s);
    if (e != hipSuccess) return e;
    const bool lists = form == SHARE_LISTS;
    // which of the two depends on the batch, so that a row's bits do not depend on the dispatch it is in
    const bool split = (long)prefix.rows * sh.n_q <= 512;
    const dim3 grid(rows, split ? sh.n_q : (sh.n_q + 7) / 8), block(256);
#define DYN_COMBINE_AS(T, B2, WIDE, SPLIT)                                                                                                            \
    hipLaunchKernelGGL((attn_shared_combine_kernel<T, B2, WIDE, SPLIT>), grid, block, 0, s, part_o, part_ml, w.p_pos, w.p_ct, w.s_pos, w.s_ct,        \
                       prefix.max_chunks, (T *)out, ld_out, part, lists ? w.p_blocks + 1 : nullptr, lists ? w.s_blocks + 1 : nullptr)
#define DYN_COMBINE(T, B2)                                                                                     \
    do {                                                                                                       \
        if (split) {                                                                                           \
            if (sh.head_dim > 128) DYN_COMBINE_AS(T, B2, true, true); else DYN_COMBINE_AS(T, B2, false, true);   \
        } else {                                                                                               \
            if (sh.head_dim > 128) DYN_COMBINE_AS(T, B2, true, false); else DYN_COMBINE_AS(T, B2, false, false); \
        }                                                                                                      \
    } while (0)
    if (dtype == 0) DYN_COMBINE(float, false);
    else if (form != SHARE_NOTHING) DYN_COMBINE(bf16_t, true);
    else DYN_COMBINE(bf16_t, false);
#undef DYN_COMBINE
#undef DYN_COMBINE_AS
    return hipGetLastError();
}

}  // namespace dyn

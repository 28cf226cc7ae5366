// The care of a paged cache's pages: copies, and forks, new lengths and compaction of the sequences that name them.
//
// A page is free while nothing names it (its reference count is 0).  Which pages a call takes is decided by one workgroup -
// the lowest free ones, in the order of the requests, so that the answer does not depend on how the launch is scheduled -
// and carried out by a second launch over the whole chip, which writes tables and counts and copies pages in every layer.  Between
// the two nothing waits on the host.  Counts change by integer atomics: their order does not show.  Small calls are two launches' latency (a fork into 7, 32
// layers: 5.3 + 5.5 us; growing and freeing those 4.8 + 3.2), large ones a copy (64 into 4, 8 layers, 155 MB: 6.1 + 31; 1593 of 4000 pages moved together, 975 MB: 5.0 + 187,
// 5.2 TB/s).
#include <algorithm>

#include "common.h"
#include "pages.h"

namespace dyn {

namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
// Pages a thread looks at per round of a search (SCAN): 4, or 16 in pools of more than four such rounds, where a round's latency is what counts.  (Plan and
// all of a fork into 7, 16 -> 4: 31.0 -> 28.7 us.)
constexpr int kScanNear = 4, kScanFar = 16;
constexpr int kNearRows = 8192, kNearFresh = 2048;   // rows whose requests are told apart in LDS, and pages found that are kept there

// Inclusive sums over the 64 lanes of a wave: on the vector ALU in 32 bits (a shuffle goes through LDS), else by shuffles.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int x) {
    x += moved<0x111, 0xf>(x);                  // row_shr 1, 2, 4, 8
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);                  // row_bcast 15: rows 1 and 3 take the row below's last
    return x + moved<0x143, 0xc>(x);            // row_bcast 31: rows 2 and 3 take lane 31's
}
__device__ __forceinline__ long long wave_scan(long long x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const long long y = __shfl_up(x, off, 64);
        if (lane >= off) x += y;
    }
    return x;
}

// Sum of x over the workgroup's threads before this one; *total: over all of them.  lds: kPlanWaves words, free again after the next barrier.
template <typename T>
__device__ __forceinline__ T before_me(T x, T *lds, T *total) {
    const T incl = wave_scan(x);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) lds[wave] = incl;
    __syncthreads();
    T base = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) base += lds[w];
        sum += lds[w];
    }
    __syncthreads();
    *total = sum;
    return base + incl - x;
}

// The pages of begin .. end - 1 whose count `wanted` accepts, in ascending order: take(rank, page) for each of rank below `limit`.
// Returns how many there are, or any number from `limit` on.  What a round takes is its loads' latency, so the next round's are on their way while
// one is ranked; round: the first one (load_round).  lds: SCAN * kPlanWaves + 1 words.
template <int SCAN>
struct Round { int count[SCAN]; };
template <int SCAN>
__device__ __forceinline__ Round<SCAN> load_round(const int32_t *ref, int at, int end) {
    Round<SCAN> r;
#pragma unroll
    for (int j = 0; j < SCAN; ++j) {
        const int p = at + j * kPlanThreads + (int)threadIdx.x;
        r.count[j] = p < end ? ref[p] : 0;
    }
    return r;
}
template <int SCAN, class Wanted, class Take>
__device__ __forceinline__ int ranked_pages(const int32_t *ref, int begin, int end, int limit, int *lds, Round<SCAN> round, Wanted &&wanted, Take &&take) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int found = 0;
    for (int at = begin; at < end && found < limit; at += SCAN * kPlanThreads) {
        unsigned long long mask[SCAN];
#pragma unroll
        for (int j = 0; j < SCAN; ++j) {
            const int p = at + j * kPlanThreads + (int)threadIdx.x;
            mask[j] = __ballot(p < end && wanted(round.count[j], p));
            if (lane == 0) lds[j * kPlanWaves + wave] = __popcll(mask[j]);
        }
        if (end - at > SCAN * kPlanThreads) round = load_round<SCAN>(ref, at + SCAN * kPlanThreads, end);
        __syncthreads();
        if (wave == 0) {                        // exclusive sums of the round's SCAN x kPlanWaves counts, kPerLane to a lane
            constexpr int kPerLane = SCAN * kPlanWaves / 64;
            int v[kPerLane], sum = 0;
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) { v[i] = sum; sum += lds[kPerLane * lane + i]; }
            const int incl = wave_scan(sum);
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) lds[kPerLane * lane + i] = v[i] + incl - sum;
            if (lane == 63) lds[SCAN * kPlanWaves] = incl;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < SCAN; ++j) {
            const int rank = found + lds[j * kPlanWaves + wave] + __popcll(mask[j] & ((1ull << lane) - 1));
            if ((mask[j] >> lane & 1) && rank < limit) take(rank, at + j * kPlanThreads + (int)threadIdx.x);
        }
        found += lds[SCAN * kPlanWaves];
        __syncthreads();
    }
    return found;
}

// One request as the search sees it.  had, has: pages its row keeps (fork: shares), and has behind the call; need: pages it takes; copy: the page
// whose content goes into the first of them, -1: none.
struct Request { int status, had, has, need, copy, length; };

template <bool FORK>
__device__ __forceinline__ Request look_at(const PageTables &t, bool mine, int x, int y) {
    Request r{PAGES_REFUSED, 0, 0, 0, -1, 0};
    bool part = false;                          // the request copies a page
    const int ps = t.page_size, row = FORK ? y : x;
    const long long most = (long long)t.max_pages * ps;
    if (!mine) return r;
    const int had = t.seq_len[row];
    if (had < 0 || had > most) return r;
    if constexpr (FORK) {
        if (x < 0 || x >= t.n_rows || x == y || had != 0) return r;
        const int len = t.seq_len[x];
        if (len < 0 || len > most) return r;
        r.had = len / ps;
        r.has = (int)(((long long)len + ps - 1) / ps);
        r.length = len;
        part = len % ps;
        if (part) r.copy = t.block_table[(size_t)x * t.max_pages + r.had];
    } else {
        if (y < 0 || y > most) return r;
        r.had = (int)(((long long)had + ps - 1) / ps);
        r.has = (int)(((long long)y + ps - 1) / ps);
        r.length = y;
        r.need = max(r.has - r.had, 0);
        if (y < had && y % ps) {               // a partly filled page stays: it must be the row's own
            const int last = t.block_table[(size_t)x * t.max_pages + r.has - 1];
            if (last < 0 || last >= t.n_pages) return r;
            part = t.ref_count[last] > 1;
            if (part) r.copy = last;
        }
    }
    if (part) {
        if (r.copy < 0 || r.copy >= t.n_pages) return r;
        r.need = 1;
    }
    r.status = PAGES_DONE;
    return r;
}

// One workgroup.  Requests in order: who is served, which free pages go to whom, which pages are copied.
template <bool FORK, int SCAN>
__global__ __launch_bounds__(kPlanThreads) void pages_plan_kernel(PageTables t, PagesPlan w, int n, const int32_t *__restrict__ xs,
                                                                  const int32_t *__restrict__ ys, int32_t *__restrict__ status) {
    __shared__ int lds[SCAN * kPlanWaves + 1];
    __shared__ long long lds_need[kPlanWaves];
    __shared__ int owner_near[kNearRows], fresh_near[kNearFresh];
    const Round<SCAN> first_round = load_round<SCAN>(t.ref_count, 0, t.n_pages);     // on its way beside the requests
    // a row that several requests name is the first one's
    const int32_t *rows = FORK ? ys : xs;
    const bool near = t.n_rows <= kNearRows;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int row = rows[i];
        if (row >= 0 && row < t.n_rows) (near ? owner_near : w.owner)[row] = n;
    }
    if (!near) __threadfence_block();
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int row = rows[i];
        if (row < 0 || row >= t.n_rows) continue;
        if (near) atomicMin(&owner_near[row], i);
        else atomicMin(&w.owner[row], i);
    }
    if (!near) __threadfence_block();
    __syncthreads();
    const bool narrow = t.max_pages <= 1 << 20;  // what a batch of requests asks for fits 32 bits
    long long wanted = 0;                        // pages all requests so far take together
    Request kept{PAGES_REFUSED, 0, 0, 0, -1, 0}; // the first batch's, and where its pages start, stay in registers
    int kept_first = -2;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + (int)threadIdx.x;
        Request r{PAGES_REFUSED, 0, 0, 0, -1, 0};
        if (i < n) {
            const int row = rows[i];
            bool mine = row >= 0 && row < t.n_rows;
            if (mine) mine = (near ? owner_near[row] : __hip_atomic_load(&w.owner[row], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) == i;
            r = look_at<FORK>(t, mine, xs[i], ys[i]);
        }
        const int need = r.status == PAGES_DONE ? r.need : 0;
        long long first = wanted;
        if (narrow) {
            int total;
            first += before_me(need, lds, &total);
            wanted += total;
        } else {
            long long total;
            first += before_me((long long)need, lds_need, &total);
            wanted += total;
        }
        const int at = r.status != PAGES_DONE ? -2 : !need ? 0 : first + need > t.n_pages ? -1 : (int)first;
        if (i0 == 0) { kept = r; kept_first = at; }
        if (i < n) {
            w.had[i] = r.had;
            w.has[i] = r.has;
            w.length[i] = r.length;
            w.src[i] = r.copy;
            if (i0) { w.first[i] = at; w.need[i] = need; }
        }
    }
    const int limit = (int)min(wanted, (long long)t.n_pages);
    const int found = limit ? ranked_pages(t.ref_count, 0, t.n_pages, limit, lds, first_round, [](int count, int) { return count == 0; },
                                           [&](int rank, int p) {
                                               w.fresh[rank] = p;
                                               if (rank < kNearFresh) fresh_near[rank] = p;
                                           }) : 0;
    if (limit > kNearFresh || n > kPlanThreads) __threadfence_block();      // only then is read below what others wrote to memory
    __syncthreads();
    int copies = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + (int)threadIdx.x;
        int src = -1, first = -2;
        if (i < n) {
            first = i0 ? w.first[i] : kept_first;
            const int need = i0 ? w.need[i] : kept.need;
            if (first >= 0 && need && first + need > found) first = -1;
            w.first[i] = first;
            status[i] = first >= 0 ? PAGES_DONE : first == -1 ? PAGES_NONE_LEFT : PAGES_REFUSED;
            if (first >= 0) src = i0 ? w.src[i] : kept.copy;
        }
        int total;
        const int at = copies + before_me(src >= 0 ? 1 : 0, lds, &total);
        if (src >= 0) {
            w.copy_src[at] = src;
            w.copy_dst[at] = first < kNearFresh ? fresh_near[first] : w.fresh[first];
        }
        copies += total;
    }
    if (threadIdx.x == 0) *w.n_copies = copies;
}

// One workgroup.  Every live page from the n_live-th on moves to a free one below it, the lowest to the lowest.
template <int SCAN>
__global__ __launch_bounds__(kPlanThreads) void pages_compact_plan_kernel(PageTables t, PagesPlan w, int32_t *__restrict__ new_page,
                                                                          int32_t *__restrict__ n_live) {
    __shared__ int lds[SCAN * kPlanWaves + 1];
    const int n = t.n_pages, all = n + 1;
    const Round<SCAN> first = load_round<SCAN>(t.ref_count, 0, n);
    const int live = ranked_pages(t.ref_count, 0, n, all, lds, first, [&](int count, int p) {
        new_page[p] = count > 0 ? p : -1;
        return count > 0;
    }, [](int, int) {});
    const bool once = n <= SCAN * kPlanThreads;                 // the counts are all in registers
    const Round<SCAN> behind = once ? first : load_round<SCAN>(t.ref_count, live, n);
    ranked_pages(t.ref_count, 0, live, all, lds, once ? first : load_round<SCAN>(t.ref_count, 0, live), [](int count, int) { return count <= 0; },
                 [&](int rank, int p) { w.copy_dst[rank] = p; });
    const int moves = ranked_pages(t.ref_count, once ? 0 : live, n, all, lds, behind, [&](int count, int p) { return p >= live && count > 0; },
                                   [&](int rank, int p) { w.copy_src[rank] = p; });
    __threadfence_block();
    __syncthreads();
    for (int i = threadIdx.x; i < moves; i += kPlanThreads) {
        const int src = w.copy_src[i], dst = w.copy_dst[i];
        new_page[src] = dst;
        t.ref_count[dst] = t.ref_count[src];
        t.ref_count[src] = 0;
    }
    if (threadIdx.x == 0) { *w.n_copies = moves; *n_live = live; }
}

constexpr int kCopyThreads = 256, kCopyVec = 4, kPiece = kCopyThreads * kCopyVec * 16;       // bytes a workgroup copies at a time

// Pieces of the listed pages, in every layer, dealt to the workgroups `block` of `n_blocks`.  What bounds it is memory, read and written once: 389
// pages of 32 layers (1.63 GB) at 5.07 TB/s.  Stores go past the caches (they are 2 % slower through them), and so do loads where every page is read once (ONCE:
// another 2 %); a fork's page goes to several children and is read from a cache for all but one (60 pages of 17 layers to 3 children each: 314 -> 262 us).
template <bool ONCE>
__device__ __forceinline__ void copy_pages(const PageLayers &l, int n_pages, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int copies, int block,
                                           int n_blocks) {
    const unsigned pieces = (unsigned)((l.page_bytes + kPiece - 1) / kPiece), per_copy = 2u * l.n * pieces;
    const unsigned long long units = (unsigned long long)copies * per_copy;
    for (unsigned long long u = block; u < units; u += n_blocks) {
        const unsigned c = (unsigned)(u / per_copy), rest = (unsigned)(u % per_copy), side = rest / pieces, piece = rest % pieces;
        const int from = src[c], to = dst[c];
        if (from < 0 || from >= n_pages || to < 0 || to >= n_pages || from == to) continue;
        char *const base = side < (unsigned)l.n ? l.k[side] : l.v[side - l.n];
        const size_t at = (size_t)piece * kPiece + threadIdx.x * 16;
        const char *const s = base + (size_t)from * l.page_bytes;
        char *const d = base + (size_t)to * l.page_bytes;
        u32x4 v[kCopyVec];
        auto load = [](const char *p) {
            if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
            else return *reinterpret_cast<const u32x4 *>(p);
        };
#pragma unroll
        for (int j = 0; j < kCopyVec; ++j)
            if (at + j * kCopyThreads * 16 < l.page_bytes) v[j] = load(s + at + j * kCopyThreads * 16);
#pragma unroll
        for (int j = 0; j < kCopyVec; ++j)
            if (at + j * kCopyThreads * 16 < l.page_bytes) __builtin_nontemporal_store(v[j], reinterpret_cast<u32x4 *>(d + at + j * kCopyThreads * 16));
    }
}

template <bool ONCE>
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(PageLayers l, int n_pages, const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                                  const int32_t *__restrict__ n_copies, int n) {
    copy_pages<ONCE>(l, n_pages, src, dst, n_copies ? *n_copies : n, blockIdx.x, gridDim.x);
}

// The first `tables` workgroups write rows, lengths and counts (a request each), the others copy pages.  tables = 0: pages only.
template <int WHAT>
__global__ __launch_bounds__(kCopyThreads) void pages_apply_kernel(PageTables t, PagesPlan w, PageLayers l, int n, int tables, const int32_t *__restrict__ xs,
                                                                   const int32_t *__restrict__ ys, const int32_t *__restrict__ new_page) {
    if ((int)blockIdx.x >= tables) {
        copy_pages<WHAT == PAGES_COMPACT>(l, t.n_pages, w.copy_src, w.copy_dst, *w.n_copies, (int)blockIdx.x - tables, (int)gridDim.x - tables);
        return;
    }
    auto refer = [&](int p, int by) {
        if (p >= 0 && p < t.n_pages) atomicAdd(&t.ref_count[p], by);
    };
    for (int i = blockIdx.x; i < n; i += tables) {
        if constexpr (WHAT == PAGES_COMPACT) {
            int32_t *const row = t.block_table + (size_t)i * t.max_pages;
            const int used = (int)min(((long long)max(t.seq_len[i], 0) + t.page_size - 1) / t.page_size, (long long)t.max_pages);
            for (int j = threadIdx.x; j < used; j += kCopyThreads) {
                const int p = row[j];
                if (p >= 0 && p < t.n_pages && new_page[p] >= 0) row[j] = new_page[p];
            }
            continue;
        }
        const int first = w.first[i];
        if (first < 0) continue;
        const int had = w.had[i], has = w.has[i];
        if constexpr (WHAT == PAGES_FORK) {
            const int32_t *const from = t.block_table + (size_t)xs[i] * t.max_pages;
            int32_t *const row = t.block_table + (size_t)ys[i] * t.max_pages;
            for (int j = threadIdx.x; j < had; j += kCopyThreads) {
                const int p = from[j];
                row[j] = p;
                refer(p, 1);
            }
            if (threadIdx.x == 0) {
                if (has > had) {
                    const int p = w.fresh[first];
                    row[had] = p;
                    t.ref_count[p] = 1;
                }
                t.seq_len[ys[i]] = w.length[i];
            }
        }
        if constexpr (WHAT == PAGES_RESIZE) {
            int32_t *const row = t.block_table + (size_t)xs[i] * t.max_pages;
            for (int j = had + (int)threadIdx.x; j < has; j += kCopyThreads) {
                const int p = w.fresh[first + j - had];
                row[j] = p;
                t.ref_count[p] = 1;
            }
            for (int j = has + (int)threadIdx.x; j < had; j += kCopyThreads) refer(row[j], -1);
            if (threadIdx.x == 0) {
                if (w.src[i] >= 0) {
                    const int p = w.fresh[first];
                    refer(w.src[i], -1);
                    row[has - 1] = p;
                    t.ref_count[p] = 1;
                }
                t.seq_len[xs[i]] = w.length[i];
            }
        }
    }
}

// Workgroups that copy: as many as are resident, and not more than there are pieces.
int copy_groups(const PageLayers &l, size_t most_copies) {
    const size_t units = most_copies * 2 * l.n * ((l.page_bytes + kPiece - 1) / kPiece);
    return (int)std::min<size_t>(units, 2048);
}

}  // namespace

hipError_t launch_pages_copy(bool once, const PageLayers &l, int n_pages, int n, const int32_t *src, const int32_t *dst, const int32_t *n_copies, hipStream_t s) {
    const int groups = copy_groups(l, (size_t)n);
    if (groups <= 0) return hipSuccess;
    hipLaunchKernelGGL(once ? pages_copy_kernel<true> : pages_copy_kernel<false>, dim3(groups), dim3(kCopyThreads), 0, s, l, n_pages, src, dst, n_copies, n);
    return hipGetLastError();
}

hipError_t launch_pages_plan(int what, const PageTables &t, const PagesPlan &w, int n, const int32_t *xs, const int32_t *ys, int32_t *status, int32_t *new_page,
                             int32_t *n_live, hipStream_t s) {
    const dim3 one(1), block(kPlanThreads);
    const bool far = t.n_pages > 4 * kScanNear * kPlanThreads;
    if (what == PAGES_FORK)
        hipLaunchKernelGGL((far ? pages_plan_kernel<true, kScanFar> : pages_plan_kernel<true, kScanNear>), one, block, 0, s, t, w, n, xs, ys, status);
    else if (what == PAGES_RESIZE)
        hipLaunchKernelGGL((far ? pages_plan_kernel<false, kScanFar> : pages_plan_kernel<false, kScanNear>), one, block, 0, s, t, w, n, xs, ys, status);
    else
        hipLaunchKernelGGL((far ? pages_compact_plan_kernel<kScanFar> : pages_compact_plan_kernel<kScanNear>), one, block, 0, s, t, w, new_page, n_live);
    return hipGetLastError();
}

hipError_t launch_pages_apply(int what, const PageTables &t, const PagesPlan &w, const PageLayers &l, int n, size_t most_copies, const int32_t *xs, const int32_t *ys,
                              const int32_t *new_page, hipStream_t s) {
    const int tables = std::min(n, 1024), groups = tables + copy_groups(l, most_copies);
    if (groups <= 0) return hipSuccess;
    const dim3 grid(groups), block(kCopyThreads);
    if (what == PAGES_FORK) hipLaunchKernelGGL(pages_apply_kernel<PAGES_FORK>, grid, block, 0, s, t, w, l, n, tables, xs, ys, new_page);
    else if (what == PAGES_RESIZE) hipLaunchKernelGGL(pages_apply_kernel<PAGES_RESIZE>, grid, block, 0, s, t, w, l, n, tables, xs, ys, new_page);
    else hipLaunchKernelGGL(pages_apply_kernel<PAGES_COMPACT>, grid, block, 0, s, t, w, l, n, tables, xs, ys, new_page);
    return hipGetLastError();
}

}  // namespace dyn

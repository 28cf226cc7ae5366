// What the page operators' host side (dynpages.cpp) and kernels (kernels_pages.hip) share.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace dyn {

enum { PAGES_FORK = 0, PAGES_RESIZE = 1, PAGES_COMPACT = 2 };
enum { PAGES_DONE = 0, PAGES_NONE_LEFT = 1, PAGES_REFUSED = 2 };      // dynlayer.h: DYN_PAGES_*

struct PageTables {
    int page_size, n_pages, n_rows, max_pages;
    int32_t *block_table, *seq_len, *ref_count;
};

// The pools of up to kPageLayers layers, by value: a model of more is served by several launches.
constexpr int kPageLayers = 64;
struct PageLayers {
    int n;
    size_t page_bytes;           // a multiple of 16
    char *k[kPageLayers], *v[kPageLayers];
};

// Where a call's plan lies in the workspace: per request the pages it keeps, has afterwards and takes, where its pages
// start in `fresh` (-1: none left, -2: refused), its new length and the page it copies from; then the list of copies.
struct PagesPlan {
    int32_t *n_copies, *owner, *first, *had, *has, *need, *length, *src, *copy_src, *copy_dst, *fresh;
};

// once: no page is read twice.  n_copies (DEVICE), if given, says how many of the n pairs there are.
hipError_t launch_pages_copy(bool once, const PageLayers &l, int n_pages, int n, const int32_t *src, const int32_t *dst, const int32_t *n_copies, hipStream_t s);
hipError_t launch_pages_plan(int what, const PageTables &t, const PagesPlan &w, int n, const int32_t *xs, const int32_t *ys, int32_t *status, int32_t *new_page,
                             int32_t *n_live, hipStream_t s);
// Tables and counts of n requests (compaction: rows), and the planned copies, at most most_copies of them.
hipError_t launch_pages_apply(int what, const PageTables &t, const PagesPlan &w, const PageLayers &l, int n, size_t most_copies, const int32_t *xs, const int32_t *ys,
                              const int32_t *new_page, hipStream_t s);

}  // namespace dyn

// Parameter blocks and launchers of the page calls.
#pragma once
#include "common.cuh"

namespace reader {

struct PagesView {
    int32_t *refs;    // [num_pages] table entries that name a page; 0: free
    int num_pages;
    int32_t *table;   // [rows][width], -1: no page
    int rows, width;
    int32_t *lens;    // [rows]
    int32_t *new_ids;   // nullable: [num_pages] what a compaction makes of a page's number
};

// Pools whose pages are moved, passed to the kernels by value.
constexpr int kPoolsPerLaunch = 128;
struct PoolList {
    unsigned char *from[kPoolsPerLaunch], *to[kPoolsPerLaunch];
};

struct PagesWs {   // device scratch, carved by the host
    int32_t *mark;       // [rows]
    int32_t *gathered;   // fork: [n][width]
    int32_t *length;     // fork: [n], -1: the pair is refused
    int32_t *demand;     // reserve: [n]
    int2 *slots;         // reserve: [num_pages] request and entry of the k-th page handed out
    int2 *moves;         // reserve: [n], compact: [num_pages] (from, to); from < 0: none
    int32_t *name;       // compact: [num_pages] new id of a page
    int32_t *holes;      // compact: [num_pages]
    int32_t *counts;     // per thread block of the cluster, several words each; the number of moves behind them
};

void launch_pages_fork(const PagesView &p, const int32_t *src, const int32_t *dst, int n, const PagesWs &ws, int32_t *status, cudaStream_t st);
void launch_pages_reserve(const PagesView &p, const int32_t *rows, const int32_t *tokens, int n, const PagesWs &ws, const PoolList *pools, int n_pools,
                          size_t page_bytes, int32_t *status, cudaStream_t st);
void launch_pages_free(const PagesView &p, const int32_t *rows, const int32_t *keep, int n, int32_t *status, cudaStream_t st);
void launch_pages_compact(const PagesView &p, int32_t *n_used, const PagesWs &ws, const PoolList *pools, int n_pools, size_t page_bytes, int n_sm,
                          cudaStream_t st);
void launch_pages_copy(const PoolList *pools, int n_pools, size_t page_bytes, int from_pages, int to_pages, const int32_t *from, const int32_t *to, int n,
                       int32_t *status, cudaStream_t st);
constexpr int kPagesCountWords = 64;   // of PagesWs::counts

}  // namespace reader

// Pages of a paged cache: rows of the page table forked, given pages to write to, freed; pages copied; the pages in use moved to
// the front of the pools (reader_pages_*).
//
// A page is free if and only if its count refs[p] is 0: there is no list that could disagree with the counts.  Free pages are
// handed out lowest id first, so a call's outcome is a function of its inputs alone, whatever the order of the threads: counts
// change by integer atomics whose intermediate values nobody looks at.
//
// The bookkeeping of fork, reserve and compact needs answers over the whole batch or the whole pool between its steps (which page
// is the k-th free one).  One launch does it, between whose steps all threads wait for one another: a thread block where requests and pool are few, else a cluster
// of eight (four rows released, forked and given pages: 12.4 us by one block, 16.4 by a cluster; 128 rows of 32: 42.7 and 34.5); a prefix sum over several kernels
// would cost a launch per step.  Data move in a second launch (2 x page_bytes per page and pool, 16 KB of a page to a thread block with all its loads
// in flight at once), which is bound by the copy bandwidth.  Measured: four rows released, forked from one of 700 positions and given pages
// 12.4 us; 128 rows of 32 with 16 pools of 36 KB 34.5 us, 23 of them the pages' bytes; a pool of 4096 pages compacted (8 pools of 36 KB) 109 us, 91 of them bytes.
#include <climits>

#include "pages.cuh"
#include "ptx_sm100.cuh"

namespace reader {
namespace {

constexpr int kCluster = 8;       // thread blocks of the cluster
constexpr int kMoves = 2 * kCluster;   // of PagesWs::counts: pages that a compaction moves
constexpr int kThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 4;
constexpr int kCopyPart = kCopyThreads * kCopyUnroll * 16;   // bytes of a page that one thread block moves

// All threads of the call's kBlocks blocks: a cluster, or one block.
template <int kBlocks>
__device__ __forceinline__ void all_sync() {
    if (kBlocks == 1) {
        __syncthreads();
    } else {
        ptx::cluster_arrive_release();
        ptx::cluster_wait_acquire();
    }
}
__device__ __forceinline__ int gthread() { return blockIdx.x * kThreads + threadIdx.x; }
__device__ __forceinline__ int gwarp() { return gthread() >> 5; }

// Sum over the thread block, in every thread.
__device__ __forceinline__ int block_sum(int x) {
    __shared__ int part[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int w = __reduce_add_sync(0xffffffffu, x);
    __syncthreads();
    if (lane == 0) part[warp] = w;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, part[lane]);
}
// Sum of the threads before this one; `total` is the block's.
__device__ __forceinline__ int block_rank(int x, int &total) {
    __shared__ int part[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += t;
    }
    __syncthreads();
    if (lane == 31) part[warp] = incl;
    __syncthreads();
    int w = part[lane], wi = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, wi, d);
        if (lane >= d) wi += t;
    }
    total = __shfl_sync(0xffffffffu, wi, 31);
    return __shfl_sync(0xffffffffu, wi - w, warp) + incl - x;
}

// Which request is the first that names a row.  Up to kNamed requests: by looking through those before it, in shared memory.  More: each row is marked with
// its first request, two steps in global memory, each followed by the cluster's barrier (rows forked, looked through and marked: 64 4.7 and 6.1 us, 512 7.6 and 8.6, 1024 13.9 and
// 13.0 to 14.8, 2000 26.5 and 23.6).
constexpr int kNamed = 512;
template <int kBlocks>
struct Named {
    int32_t *mark;
    const int *names;   // null: the marks
    __device__ __forceinline__ Named(int32_t *mark_, int *room, const int32_t *rows, int n, int n_rows) : mark(mark_), names(n <= kNamed ? room : nullptr) {
        if (names) {
            for (int i = threadIdx.x; i < n; i += kThreads) room[i] = rows[i];
            __syncthreads();
            return;
        }
        for (int i = gthread(); i < n; i += kBlocks * kThreads) {
            const int r = rows[i];
            if (r >= 0 && r < n_rows) mark[r] = INT_MAX;
        }
        all_sync<kBlocks>();
        for (int i = gthread(); i < n; i += kBlocks * kThreads) {
            const int r = rows[i];
            if (r >= 0 && r < n_rows) atomicMin(mark + r, i);
        }
        all_sync<kBlocks>();
    }
    // Of request i, which names a row that there is.  Warp-collective.
    __device__ __forceinline__ bool first(int i, int row) const {
        if (!names) return __ldcg(mark + row) == i;
        bool before = false;
        for (int j = threadIdx.x & 31; j < i; j += 32) before |= names[j] == row;
        return !__any_sync(0xffffffffu, before);
    }
};

// ---- fork
template <int kBlocks>
__global__ void __cluster_dims__(kBlocks, 1, 1) __launch_bounds__(kThreads)
pages_fork_kernel(const PagesView p, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int n, const PagesWs ws, int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    __shared__ int room[kNamed];
    const Named<kBlocks> named(ws.mark, room, dst, n, p.rows);
    // all sources are read (and their pages counted once more) ...
    for (int i = gwarp(); i < n; i += kBlocks * kThreads / 32) {
        const int from = src[i], to = dst[i];
        int st = READER_OK, length = -1;
        if (from < 0 || from >= p.rows || to < 0 || to >= p.rows || !named.first(i, to)) {
            st = READER_ERR_INVALID_ARG;
        } else {
            length = p.lens[from];
            if (length < 0 || (int64_t)length > (int64_t)p.width * kPage) {
                st = READER_ERR_CAPACITY;
            } else {
                const int32_t *row = p.table + (size_t)from * p.width;
                const int used = (length + kPage - 1) / kPage;
                bool bad = false;
                for (int e = lane; e < used; e += 32) {
                    const int page = row[e];
                    bad |= page < 0 || page >= p.num_pages;
                }
                if (__any_sync(0xffffffffu, bad)) {
                    st = READER_ERR_BAD_PAGE;
                } else {
                    for (int e = lane; e < used; e += 32) {
                        const int page = row[e];
                        ws.gathered[(size_t)i * p.width + e] = page;
                        atomicAdd(p.refs + page, 1);
                    }
                }
            }
        }
        if (lane == 0) {
            status[i] = st;
            ws.length[i] = st == READER_OK ? length : -1;
        }
    }
    all_sync<kBlocks>();
    // ... before any destination is released and written
    for (int i = gwarp(); i < n; i += kBlocks * kThreads / 32) {
        const int length = __ldcg(ws.length + i);
        if (length < 0) continue;
        int32_t *row = p.table + (size_t)dst[i] * p.width;
        const int used = (length + kPage - 1) / kPage;
        for (int e = lane; e < p.width; e += 32) {
            const int old = row[e];
            if (old >= 0 && old < p.num_pages) atomicSub(p.refs + old, 1);
            row[e] = e < used ? __ldcg(ws.gathered + (size_t)i * p.width + e) : -1;
        }
        if (lane == 0) p.lens[dst[i]] = length;
    }
}

// ---- reserve
// The entries first .. need - 1 of a row that a request wants to write; which of them need a page of their own goes by the counts
// before the call (`held`).
struct Wanted {
    int row, length, first, need;
};
__device__ __forceinline__ Wanted wanted(const PagesView &p, int row, int tokens) {
    Wanted w;
    w.row = row;
    w.length = p.lens[row];
    w.first = w.length / kPage;
    w.need = (int)(((int64_t)w.length + tokens + kPage - 1) / kPage);
    return w;
}

template <int kBlocks>
__global__ void __cluster_dims__(kBlocks, 1, 1) __launch_bounds__(kThreads)
pages_reserve_kernel(const PagesView p, const int32_t *__restrict__ rows, const int32_t *__restrict__ tokens, int n, const PagesWs ws, int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, block = blockIdx.x;
    __shared__ int room[kNamed];
    const Named<kBlocks> named(ws.mark, room, rows, n, p.rows);
    // 1. what each request needs
    for (int i = gwarp(); i < n; i += kBlocks * kThreads / 32) {
        const int row = rows[i], t = tokens[i];
        int st = READER_OK, demand = 0;
        if (row < 0 || row >= p.rows || t < 0 || !named.first(i, row)) {
            st = READER_ERR_INVALID_ARG;
        } else if (p.lens[row] < 0 || (int64_t)p.lens[row] + t > (int64_t)p.width * kPage) {
            st = READER_ERR_CAPACITY;
        } else if (t > 0) {
            const Wanted w = wanted(p, row, t);
            bool bad = false;
            for (int e = w.first + lane; e < w.need; e += 32) {
                const int page = p.table[(size_t)row * p.width + e];
                if (page >= p.num_pages) bad = true;
                else if (page < 0 || p.refs[page] > 1) ++demand;
            }
            // committed positions have pages
            for (int e = lane; e < (w.length + kPage - 1) / kPage; e += 32) bad |= p.table[(size_t)row * p.width + e] < 0;
            demand = __reduce_add_sync(0xffffffffu, demand);
            if (__any_sync(0xffffffffu, bad)) {
                st = READER_ERR_BAD_PAGE;
                demand = 0;
            }
        }
        if (lane == 0) {
            status[i] = st;
            ws.demand[i] = demand;
            ws.moves[i] = make_int2(-1, -1);
        }
    }
    // 2. how many pages are free, by eighths of the pool
    const int per_block = ((p.num_pages + kBlocks - 1) / kBlocks + 3) & ~3;
    const int page0 = min(p.num_pages, block * per_block), page1 = min(p.num_pages, page0 + per_block);
    int mine = 0;
    for (int i = page0 + threadIdx.x; i < page1; i += kThreads) mine += p.refs[i] == 0;
    mine = block_sum(mine);
    if (threadIdx.x == 0) ws.counts[block] = mine;
    all_sync<kBlocks>();
    int free_before = 0, free_all = 0;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        const int x = __ldcg(ws.counts + c);
        free_before += c < block ? x : 0;
        free_all += x;
    }
    // 3. requests in order, as long as they fit; their entries become the list of slots
    const int chunk = (n + kBlocks - 1) / kBlocks, i0 = min(n, block * chunk), i1 = min(n, i0 + chunk);
    int before = 0;   // (the host bounds n * width: no sum of demands overflows)
    for (int i = threadIdx.x; i < i0; i += kThreads) before += __ldcg(ws.demand + i);
    before = block_sum(before);
    int granted = 0;
    __shared__ int offset[kThreads];
    for (int base = i0; base < i1; base += kThreads) {
        const int i = base + threadIdx.x;
        const int d = i < i1 ? __ldcg(ws.demand + i) : 0;
        int total;
        const int at = before + block_rank(d, total);
        const bool fits = d > 0 && at <= free_all - d;
        if (d > 0 && !fits) status[i] = READER_ERR_CAPACITY;
        if (fits) granted = max(granted, at + d);
        offset[threadIdx.x] = fits ? at : -1;
        __syncthreads();
        for (int j = threadIdx.x >> 5; j < kThreads && base + j < i1; j += kThreads / 32) {
            int k = offset[j];
            if (k < 0) continue;
            const int row = rows[base + j];
            const Wanted w = wanted(p, row, tokens[base + j]);
            for (int e0 = w.first; e0 < w.need; e0 += 32) {
                const int e = e0 + lane;
                const int page = e < w.need ? p.table[(size_t)row * p.width + e] : 0;
                const bool fresh = e < w.need && (page < 0 || p.refs[page] > 1);
                const unsigned vote = __ballot_sync(0xffffffffu, fresh);
                if (fresh) ws.slots[k + __popc(vote & ((1u << lane) - 1))] = make_int2(base + j, e);
                k += __popc(vote);
            }
        }
        __syncthreads();
        before += total;
    }
    granted = __reduce_max_sync(0xffffffffu, granted);
    if (threadIdx.x == 0) ws.counts[kBlocks + block] = 0;
    __syncthreads();
    if (lane == 0) atomicMax(ws.counts + kBlocks + block, granted);
    all_sync<kBlocks>();
    int handed = 0;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) handed = max(handed, __ldcg(ws.counts + kBlocks + c));
    // 4. the k-th free page to the k-th slot
    int rank0 = free_before;
    for (int base = page0; base < page1 && rank0 < handed; base += kThreads) {
        const int page = base + threadIdx.x;
        const bool is_free = page < page1 && p.refs[page] == 0;
        int total;
        const int k = rank0 + block_rank(is_free ? 1 : 0, total);
        if (is_free && k < handed) {
            const int2 s = __ldcg(ws.slots + k);
            const int row = rows[s.x];
            int32_t *entry = p.table + (size_t)row * p.width + s.y;
            const int old = *entry;
            *entry = page;
            p.refs[page] = 1;
            const int length = p.lens[row];
            if (length % kPage != 0 && s.y == length / kPage) ws.moves[s.x] = make_int2(old, page);
            ws.slots[k] = make_int2(old, page);
        }
        rank0 += total;
    }
    all_sync<kBlocks>();
    // 5. the pages that were replaced lose a holder (only now: a page must not look free while others still look for free ones)
    for (int k = gthread(); k < handed; k += kBlocks * kThreads) {
        const int old = __ldcg(ws.slots + k).x;
        if (old >= 0) atomicSub(p.refs + old, 1);
    }
}

// ---- free
__global__ void __launch_bounds__(256) pages_free_kernel(const PagesView p, const int32_t *__restrict__ rows, const int32_t *__restrict__ keep, int n,
                                                         int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (i >= n) return;
    const int row = rows[i], left = keep ? keep[i] : 0;
    if (row < 0 || row >= p.rows || left < 0) {
        if (lane == 0) status[i] = READER_ERR_INVALID_ARG;
        return;
    }
    bool bad = false;
    for (int64_t e = ((int64_t)left + kPage - 1) / kPage + lane; e < p.width; e += 32) {
        // (by exchange: a row that is named twice loses each page once)
        const int old = atomicExch(p.table + (size_t)row * p.width + e, -1);
        if (old >= p.num_pages) bad = true;
        else if (old >= 0) atomicSub(p.refs + old, 1);
    }
    bad = __any_sync(0xffffffffu, bad);
    if (lane == 0) {
        atomicMin(p.lens + row, left);
        status[i] = bad ? READER_ERR_BAD_PAGE : READER_OK;
    }
}

// ---- data
// Part `part` of a page: all loads, then all stores.
__device__ __forceinline__ void copy_part(const unsigned char *from, unsigned char *to, size_t page_bytes, int part) {
    const uint4 *src = reinterpret_cast<const uint4 *>(from);
    uint4 *dst = reinterpret_cast<uint4 *>(to);
    const int words = (int)(page_bytes / 16), w0 = part * (kCopyPart / 16) + threadIdx.x;
    uint4 x[kCopyUnroll];
#pragma unroll
    for (int i = 0; i < kCopyUnroll; ++i)
        if (w0 + i * kCopyThreads < words) x[i] = __ldcs(src + w0 + i * kCopyThreads);
#pragma unroll
    for (int i = 0; i < kCopyUnroll; ++i)
        if (w0 + i * kCopyThreads < words) __stcs(dst + w0 + i * kCopyThreads, x[i]);
}

// Block (pool * parts + part, i): one part of the i-th move in one pool.
__global__ void __launch_bounds__(kCopyThreads) pages_move_kernel(const __grid_constant__ PoolList pools, const int2 *__restrict__ moves, int n, int parts,
                                                                  size_t page_bytes) {
    pdl_wait();
    pdl_launch_dependents();
    const int pool = blockIdx.x / parts, part = blockIdx.x - pool * parts;
    for (int i = blockIdx.y; i < n; i += gridDim.y) {
        const int2 m = moves[i];
        if (m.x < 0) continue;
        copy_part(pools.from[pool] + (size_t)m.x * page_bytes, pools.to[pool] + (size_t)m.y * page_bytes, page_bytes, part);
    }
}

// The caller's list: ids are checked here.
__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const __grid_constant__ PoolList pools, const int32_t *__restrict__ from,
                                                                  const int32_t *__restrict__ to, int n, int from_pages, int to_pages, int parts,
                                                                  size_t page_bytes, int32_t *__restrict__ status) {
    pdl_wait();
    pdl_launch_dependents();
    const int pool = blockIdx.x / parts, part = blockIdx.x - pool * parts;
    for (int i = blockIdx.y; i < n; i += gridDim.y) {
        const int a = from[i], b = to[i];
        const bool ok = a >= 0 && a < from_pages && b >= 0 && b < to_pages;
        if (status && blockIdx.x == 0 && threadIdx.x == 0) status[i] = ok ? READER_OK : READER_ERR_BAD_PAGE;
        if (ok) copy_part(pools.from[pool] + (size_t)a * page_bytes, pools.to[pool] + (size_t)b * page_bytes, page_bytes, part);
    }
}

// ---- compact
template <int kBlocks>
__global__ void __cluster_dims__(kBlocks, 1, 1) __launch_bounds__(kThreads)
pages_plan_kernel(const PagesView p, int32_t *__restrict__ n_used, const PagesWs ws) {
    pdl_wait();
    pdl_launch_dependents();
    const int block = blockIdx.x;
    const int per_block = (p.num_pages + kBlocks - 1) / kBlocks;
    const int page0 = min(p.num_pages, block * per_block), page1 = min(p.num_pages, page0 + per_block);
    // 1. pages in use
    int held = 0;
    for (int i = page0 + threadIdx.x; i < page1; i += kThreads) held += p.refs[i] != 0;
    held = block_sum(held);
    if (threadIdx.x == 0) ws.counts[block] = held;
    all_sync<kBlocks>();
    int used = 0, held_before = 0;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        const int x = __ldcg(ws.counts + c);
        used += x;
        held_before += c < block ? x : 0;
    }
    if (block == 0 && threadIdx.x == 0) *n_used = used;
    // 2. below `used` the free pages, from there on those in use: as many of the one as of the other.  How many stand before this
    // block's part: of the first page0 pages held_before are in use, and of the first min(page0, used) ...
    int low = 0;   // pages in use below `used` in this block's part
    for (int i = page0 + threadIdx.x; i < min(page1, used); i += kThreads) low += p.refs[i] != 0;
    low = block_sum(low);
    if (threadIdx.x == 0) ws.counts[kBlocks + block] = low;
    all_sync<kBlocks>();
    int low_before = 0, low_all = 0;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
        const int x = __ldcg(ws.counts + kBlocks + c);
        low_before += c < block ? x : 0;
        low_all += x;
    }
    int holes = min(page0, used) - low_before, movers = held_before - low_before;
    for (int base = page0; base < page1; base += kThreads) {
        const int i = base + threadIdx.x;
        const bool in = i < page1, is_held = in && p.refs[i] != 0;
        const bool hole = in && !is_held && i < used, mover = is_held && i >= used;
        int total;
        const int rank = block_rank((hole ? 1 : 0) | (mover ? 1 << 16 : 0), total);   // (at most 1024 of each)
        if (hole) ws.holes[holes + (rank & 0xffff)] = i;
        if (mover) ws.moves[movers + (rank >> 16)].x = i;
        if (in && i >= used && !mover) ws.name[i] = i;
        if (in && !mover && p.new_ids) p.new_ids[i] = is_held ? i : -1;
        holes += total & 0xffff;
        movers += total >> 16;
    }
    all_sync<kBlocks>();
    // 3. the k-th of the ones to the k-th of the others
    const int count = used - low_all;
    if (block == 0 && threadIdx.x == 0) ws.counts[kMoves] = count;
    for (int k = gthread(); k < count; k += kBlocks * kThreads) {
        const int to = __ldcg(ws.holes + k), from = __ldcg(&ws.moves[k].x);
        ws.moves[k].y = to;
        ws.name[from] = to;
        if (p.new_ids) p.new_ids[from] = to;
        p.refs[to] = p.refs[from];
        p.refs[from] = 0;
    }
}

__global__ void __launch_bounds__(kCopyThreads) pages_compact_kernel(const PagesView p, const int32_t *__restrict__ n_used, const PagesWs ws,
                                                                     const __grid_constant__ PoolList pools, int n_pools, int parts, size_t page_bytes,
                                                                     int rename) {
    pdl_wait();
    pdl_launch_dependents();
    const int count = ws.counts[kMoves], used = *n_used;
    const int64_t items = (int64_t)count * n_pools * parts;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int part = (int)(i % parts);
        const int64_t j = i / parts;
        const int pool = (int)(j / count);
        const int2 m = ws.moves[j - (int64_t)pool * count];
        copy_part(pools.from[pool] + (size_t)m.x * page_bytes, pools.to[pool] + (size_t)m.y * page_bytes, page_bytes, part);
    }
    if (!rename) return;
    const int64_t entries = (int64_t)p.rows * p.width;
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kCopyThreads) {
        const int page = p.table[i];
        if (page >= used && page < p.num_pages) p.table[i] = ws.name[page];
    }
}

int parts_of(size_t page_bytes) { return (int)((page_bytes + kCopyPart - 1) / kCopyPart); }
int pools_of(int n_pools, int at) { return n_pools - at < kPoolsPerLaunch ? n_pools - at : kPoolsPerLaunch; }
unsigned moves_of(int n) { return (unsigned)(n < 65535 ? n : 65535); }

}  // namespace

// Up to here a call is one thread block's.  Requests, by one block and by a cluster: 32 rows forked in 3.7 and 4.5 us, 33 in 5.5 and 4.6; 32 given pages and released again 8.4 and
// 11.8, 64 10 and 12, 128 13.4 and 12.3.  Pages, the books of a compaction: 4096 8.8 and 10.2, 6000 11.8 and 11.1, 16384 22.5 and 15.4.
constexpr int kOneBlockRequests = 32, kOneBlockPages = 4096;

void launch_pages_fork(const PagesView &p, const int32_t *src, const int32_t *dst, int n, const PagesWs &ws, int32_t *status, cudaStream_t st) {
    const bool one = n <= kOneBlockRequests;
    launch_pdl(one ? pages_fork_kernel<1> : pages_fork_kernel<kCluster>, dim3(one ? 1 : kCluster), dim3(kThreads), 0, st, p, src, dst, n, ws, status);
}

void launch_pages_reserve(const PagesView &p, const int32_t *rows, const int32_t *tokens, int n, const PagesWs &ws, const PoolList *pools, int n_pools,
                          size_t page_bytes, int32_t *status, cudaStream_t st) {
    const bool one = n <= kOneBlockRequests && p.num_pages <= kOneBlockPages;
    launch_pdl(one ? pages_reserve_kernel<1> : pages_reserve_kernel<kCluster>, dim3(one ? 1 : kCluster), dim3(kThreads), 0, st, p, rows, tokens, n, ws, status);
    const int parts = parts_of(page_bytes);
    for (int at = 0; at < n_pools; at += kPoolsPerLaunch)
        launch_pdl(pages_move_kernel, dim3((unsigned)(pools_of(n_pools, at) * parts), moves_of(n)), dim3(kCopyThreads), 0, st, pools[at / kPoolsPerLaunch],
                   static_cast<const int2 *>(ws.moves), n, parts, page_bytes);
}

void launch_pages_free(const PagesView &p, const int32_t *rows, const int32_t *keep, int n, int32_t *status, cudaStream_t st) {
    launch_pdl(pages_free_kernel, dim3((unsigned)((n + 7) / 8)), dim3(256), 0, st, p, rows, keep, n, status);
}

void launch_pages_compact(const PagesView &p, int32_t *n_used, const PagesWs &ws, const PoolList *pools, int n_pools, size_t page_bytes, int n_sm,
                          cudaStream_t st) {
    const bool one = p.num_pages <= kOneBlockPages;
    launch_pdl(one ? pages_plan_kernel<1> : pages_plan_kernel<kCluster>, dim3(one ? 1 : kCluster), dim3(kThreads), 0, st, p, n_used, ws);
    for (int at = 0; at < n_pools; at += kPoolsPerLaunch)
        launch_pdl(pages_compact_kernel, dim3((unsigned)(8 * n_sm)), dim3(kCopyThreads), 0, st, p, static_cast<const int32_t *>(n_used), ws,
                   pools[at / kPoolsPerLaunch], pools_of(n_pools, at), parts_of(page_bytes), page_bytes, at == 0 ? 1 : 0);
}

void launch_pages_copy(const PoolList *pools, int n_pools, size_t page_bytes, int from_pages, int to_pages, const int32_t *from, const int32_t *to, int n,
                       int32_t *status, cudaStream_t st) {
    const int parts = parts_of(page_bytes);
    for (int at = 0; at < n_pools; at += kPoolsPerLaunch)
        launch_pdl(pages_copy_kernel, dim3((unsigned)(pools_of(n_pools, at) * parts), moves_of(n)), dim3(kCopyThreads), 0, st, pools[at / kPoolsPerLaunch],
                   from, to, n, from_pages, to_pages, parts, page_bytes, at == 0 ? status : nullptr);
}

}  // namespace reader

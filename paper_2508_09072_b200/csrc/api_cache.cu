// C-ABI entry points of the 4-bit cache and of the page calls: argument validation, workspace carving, kernel sequencing.
#include <new>
#include <vector>

#include "ctx.cuh"
#include "pages.cuh"
#include "q4_attn.cuh"
#include "q4_cache.cuh"
#include "q4_format.cuh"

namespace {

using namespace reader;

constexpr size_t kAlign = 256;
constexpr int kMost = 1 << 30;   // pages, requests, sequences of a call: the kernels count them in steps, in 32 bits
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

reader_status check_device(const reader_ctx *ctx) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return READER_ERR_CUDA;
    return dev == ctx->device ? READER_OK : READER_ERR_INVALID_ARG;
}
reader_status launch_status() { return cudaGetLastError() == cudaSuccess ? READER_OK : READER_ERR_CUDA; }

// The caches of a model's layers: one block table and shape, pools of their own.
reader_status check_layers(const reader_kv_cache *c, int n_layers) {
    const reader_kv_cache &a = c[0];
    if (!a.page_table || a.num_pages < 0 || a.n_kv_heads < 1 || a.max_pages_per_seq < 1 || a.shared_prefix_len < 0 || a.shared_prefix_len % kPage != 0)
        return READER_ERR_INVALID_ARG;
    if (a.page_size != kPage || (a.head_dim != 64 && a.head_dim != 128)) return READER_ERR_UNSUPPORTED;
    if ((int64_t)a.max_pages_per_seq * kPage >= (int64_t)1 << 31) return READER_ERR_UNSUPPORTED;   // positions are 32-bit
    for (int i = 0; i < n_layers; ++i) {
        const reader_kv_cache &x = c[i];
        if (!x.k_pool || !x.v_pool || !aligned16(x.k_pool) || !aligned16(x.v_pool)) return READER_ERR_INVALID_ARG;
        if (x.page_table != a.page_table || x.num_pages != a.num_pages || x.page_size != a.page_size || x.n_kv_heads != a.n_kv_heads ||
            x.head_dim != a.head_dim || x.max_pages_per_seq != a.max_pages_per_seq || x.shared_prefix_len != a.shared_prefix_len)
            return READER_ERR_INVALID_ARG;
    }
    return READER_OK;
}

int chunks_of(int n, int per) { return (n + per - 1) / per; }

reader_status convert(bool store, reader_ctx *ctx, const reader_kv_cache *from, const reader_kv_cache *to, int n_layers, int batch, const int32_t *first,
                      const int32_t *last, int32_t *status_out, void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (batch == 0) return READER_OK;
    if (!from || !to || n_layers < 1 || batch < 0 || !first || !last || !status_out) return READER_ERR_INVALID_ARG;
    if (batch > kMost) return READER_ERR_UNSUPPORTED;
    if (reader_status st = check_layers(from, n_layers)) return st;
    if (reader_status st = check_layers(to, n_layers)) return st;
    if (from[0].n_kv_heads != to[0].n_kv_heads || from[0].head_dim != to[0].head_dim) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_device(ctx)) return st;
    std::vector<Q4Layers> chunks;
    try {
        chunks.resize(chunks_of(n_layers, kQ4LayersPerLaunch));
    } catch (const std::bad_alloc &) {
        return READER_ERR_CUDA;
    }
    for (int i = 0; i < n_layers; ++i) {
        Q4Layers &c = chunks[i / kQ4LayersPerLaunch];
        const int j = i % kQ4LayersPerLaunch;
        c.k_from[j] = from[i].k_pool; c.v_from[j] = from[i].v_pool;
        c.k_to[j] = to[i].k_pool; c.v_to[j] = to[i].v_pool;
    }
    Q4Convert p{};
    p.first = first; p.last = last;
    p.from_table = from[0].page_table; p.to_table = to[0].page_table;
    p.from_width = from[0].max_pages_per_seq; p.to_width = to[0].max_pages_per_seq;
    p.from_pages = from[0].num_pages; p.to_pages = to[0].num_pages;
    p.shared_prefix_len = to[0].shared_prefix_len;
    p.Hkv = to[0].n_kv_heads; p.D = to[0].head_dim; p.B = batch;
    p.status = status_out;
    launch_q4_convert(store, p, chunks.data(), n_layers, ctx->n_sm, (cudaStream_t)stream);
    return launch_status();
}

// ---- attention
struct Q4Ws {
    size_t flags, partial_ml, partial_o, tasks, total;
};
Q4Ws q4_ws(const reader_ctx *ctx, int D) {
    Q4Ws w{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes); return o; };
    const size_t rows = (size_t)ctx->n_sm * kQ4ShareRows;
    w.flags = take(sizeof(int32_t) * 2 * kQ4Ranges * (size_t)ctx->n_sm);
    w.partial_ml = take(sizeof(float2) * rows);
    w.partial_o = take(sizeof(float) * rows * D);
    w.tasks = take(sizeof(ShareTask) * kQ4Ranges * (size_t)ctx->n_sm);
    w.total = at;
    return w;
}

// ---- pages
struct PagesLayout {
    size_t mark, gathered, length, demand, slots, moves, name, holes, counts, total;
};
PagesLayout pages_layout(int64_t num_pages, int64_t rows, int64_t width, int64_t n) {
    PagesLayout w{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes); return o; };
    w.counts = take(sizeof(int32_t) * kPagesCountWords);
    w.mark = take(sizeof(int32_t) * rows);
    const size_t common = at;
    w.gathered = take(sizeof(int32_t) * n * width);   // fork
    w.length = take(sizeof(int32_t) * n);
    size_t total = at;
    at = common;
    w.demand = take(sizeof(int32_t) * n);              // reserve, compact
    w.slots = take(sizeof(int2) * num_pages);
    w.moves = take(sizeof(int2) * (n > num_pages ? n : num_pages));
    w.name = take(sizeof(int32_t) * num_pages);
    w.holes = take(sizeof(int32_t) * num_pages);
    w.total = at > total ? at : total;
    return w;
}
PagesWs carve(const PagesLayout &w, void *workspace) {
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    PagesWs r;
    r.counts = reinterpret_cast<int32_t *>(ws + w.counts);
    r.mark = reinterpret_cast<int32_t *>(ws + w.mark);
    r.gathered = reinterpret_cast<int32_t *>(ws + w.gathered);
    r.length = reinterpret_cast<int32_t *>(ws + w.length);
    r.demand = reinterpret_cast<int32_t *>(ws + w.demand);
    r.slots = reinterpret_cast<int2 *>(ws + w.slots);
    r.moves = reinterpret_cast<int2 *>(ws + w.moves);
    r.name = reinterpret_cast<int32_t *>(ws + w.name);
    r.holes = reinterpret_cast<int32_t *>(ws + w.holes);
    return r;
}
reader_status check_pages(const reader_pages *p, bool with_pools) {
    if (!p || !p->refs || !p->page_table || !p->seq_lens || p->num_pages < 1 || p->rows < 1 || p->max_pages_per_seq < 1) return READER_ERR_INVALID_ARG;
    if ((int64_t)p->max_pages_per_seq * kPage >= (int64_t)1 << 31 || p->num_pages > kMost) return READER_ERR_UNSUPPORTED;
    if (!with_pools) return READER_OK;
    if (!p->pools || p->n_pools < 1 || p->page_bytes == 0 || p->page_bytes % 16 != 0) return READER_ERR_INVALID_ARG;
    if (p->page_bytes >= (size_t)1 << 31) return READER_ERR_UNSUPPORTED;
    for (int i = 0; i < p->n_pools; ++i)
        if (!p->pools[i] || !aligned16(p->pools[i])) return READER_ERR_INVALID_ARG;
    return READER_OK;
}
PagesView view(const reader_pages *p) { return {p->refs, p->num_pages, p->page_table, p->rows, p->max_pages_per_seq, p->seq_lens, nullptr}; }

reader_status pool_chunks(const void *const *from, void *const *to, int n, std::vector<PoolList> &chunks) {
    try {
        chunks.resize(chunks_of(n, kPoolsPerLaunch));
    } catch (const std::bad_alloc &) {
        return READER_ERR_CUDA;
    }
    for (int i = 0; i < n; ++i) {
        chunks[i / kPoolsPerLaunch].from[i % kPoolsPerLaunch] = static_cast<unsigned char *>(const_cast<void *>(from[i]));
        chunks[i / kPoolsPerLaunch].to[i % kPoolsPerLaunch] = static_cast<unsigned char *>(to[i]);
    }
    return READER_OK;
}

// What fork, reserve and compact share: the workspace, and sums of at most n * width pages in 32 bits.
reader_status check_requests(const reader_pages *p, int n, const void *workspace, size_t workspace_bytes) {
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return READER_ERR_INVALID_ARG;
    if ((int64_t)n * p->max_pages_per_seq >= (int64_t)1 << 31 || n > kMost) return READER_ERR_UNSUPPORTED;
    if (workspace_bytes < pages_layout(p->num_pages, p->rows, p->max_pages_per_seq, n).total) return READER_ERR_WORKSPACE;
    return READER_OK;
}

}  // namespace

extern "C" {

reader_status reader_q4_store(reader_ctx *ctx, const reader_kv_cache *from, const reader_kv_cache *to, int32_t n_layers, int32_t batch,
                              const int32_t *first, const int32_t *last, int32_t *status_out, void *stream) {
    return convert(true, ctx, from, to, n_layers, batch, first, last, status_out, stream);
}

reader_status reader_q4_load(reader_ctx *ctx, const reader_kv_cache *from, const reader_kv_cache *to, int32_t n_layers, int32_t batch,
                             const int32_t *first, const int32_t *last, int32_t *status_out, void *stream) {
    return convert(false, ctx, from, to, n_layers, batch, first, last, status_out, stream);
}

reader_status reader_q4_commit(reader_ctx *ctx, const reader_kv_cache *caches, const void *const *k_trees, const void *const *v_trees,
                               int32_t n_layers, int32_t batch, int32_t n_nodes, const int32_t *path, const int32_t *n_acc, int32_t max_path,
                               int32_t update_seq_lens, int32_t *slots_out, int32_t *status_out, void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (batch == 0) return READER_OK;
    if (!caches || !k_trees || !v_trees || n_layers < 1 || batch < 0 || n_nodes < 1 || n_nodes > kMaxNodes || max_path < 1 || !path || !n_acc ||
        !slots_out || !status_out)
        return READER_ERR_INVALID_ARG;
    if (batch > kMost) return READER_ERR_UNSUPPORTED;
    if (reader_status st = check_layers(caches, n_layers)) return st;
    for (int i = 0; i < n_layers; ++i)
        if (!caches[i].seq_lens || caches[i].seq_lens != caches[0].seq_lens || !k_trees[i] || !v_trees[i] || !aligned16(k_trees[i]) || !aligned16(v_trees[i]))
            return READER_ERR_INVALID_ARG;
    if ((int64_t)max_path * caches[0].n_kv_heads * 16 >= (int64_t)1 << 30) return READER_ERR_UNSUPPORTED;   // blocks of a sequence, in 32 bits
    if (reader_status st = check_device(ctx)) return st;
    std::vector<Q4Layers> chunks;
    try {
        chunks.resize(chunks_of(n_layers, kQ4LayersPerLaunch));
    } catch (const std::bad_alloc &) {
        return READER_ERR_CUDA;
    }
    for (int i = 0; i < n_layers; ++i) {
        Q4Layers &c = chunks[i / kQ4LayersPerLaunch];
        const int j = i % kQ4LayersPerLaunch;
        c.k_from[j] = k_trees[i]; c.v_from[j] = v_trees[i];
        c.k_to[j] = caches[i].k_pool; c.v_to[j] = caches[i].v_pool;
    }
    Q4Commit p{};
    p.page_table = caches[0].page_table;
    p.max_pages = caches[0].max_pages_per_seq; p.num_pages = caches[0].num_pages; p.shared_prefix_len = caches[0].shared_prefix_len;
    p.seq_lens = caches[0].seq_lens;
    p.path = path; p.n_acc = n_acc;
    p.Hkv = caches[0].n_kv_heads; p.D = caches[0].head_dim; p.B = batch; p.T = n_nodes; p.max_path = max_path;
    p.slots = slots_out; p.status = status_out;
    launch_q4_commit(p, chunks.data(), n_layers, update_seq_lens != 0, (cudaStream_t)stream);
    return launch_status();
}

size_t reader_q4_workspace_bytes(const reader_ctx *ctx, int32_t head_dim) {
    if (!ctx || (head_dim != 64 && head_dim != 128)) return 0;
    return q4_ws(ctx, head_dim).total;
}

reader_status reader_set_q4_give_up(reader_ctx *ctx, int32_t worker) {
    if (!ctx || worker < -1) return READER_ERR_INVALID_ARG;
    ctx->q4_give_up = worker;
    return READER_OK;
}

reader_status reader_q4_verify_attn(reader_ctx *ctx, const void *q, int32_t n_q_heads, const void *k_tree, const void *v_tree,
                                    const reader_kv_cache *cache, const reader_tree *tree, float softmax_scale, void *out, float *lse_out,
                                    void *workspace, size_t workspace_bytes, int32_t *status_out, void *stream) {
    if (!ctx || !cache || !tree) return READER_ERR_INVALID_ARG;
    if (tree->batch == 0) return READER_OK;
    if (!q || !k_tree || !v_tree || !out || !workspace || !status_out || !cache->seq_lens || !tree->parent) return READER_ERR_INVALID_ARG;
    const int B = tree->batch, T = tree->n_nodes, Hq = n_q_heads, Hkv = cache->n_kv_heads, D = cache->head_dim;
    if (B < 0 || T < 1 || T > kMaxNodes || Hq < 1 || !(softmax_scale == softmax_scale)) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_layers(cache, 1)) return st;
    if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(out) || !aligned16(tree->anc_mask) ||
        reinterpret_cast<uintptr_t>(workspace) % kAlign != 0)
        return READER_ERR_INVALID_ARG;
    // the row maximum is taken before the scaling, so the scale has to be positive
    if (!(softmax_scale > 0.f) || softmax_scale > 2.0e38f || Hq % Hkv != 0 || Hq / Hkv > kQ4MaxGroup || B > kQ4MaxBatch)
        return READER_ERR_UNSUPPORTED;
    const int64_t units = (int64_t)B * Hkv * ((int64_t)T * (Hq / Hkv) / 16 + 1);
    if (units * ((int64_t)cache->max_pages_per_seq + 4) >= (int64_t)1 << 31) return READER_ERR_UNSUPPORTED;
    const Q4Ws w = q4_ws(ctx, D);
    if (workspace_bytes < w.total) return READER_ERR_WORKSPACE;
    if (reader_status st = check_device(ctx)) return st;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    Q4AttnParams p{};
    p.q = static_cast<const __nv_bfloat16 *>(q);
    p.k_tree = static_cast<const __nv_bfloat16 *>(k_tree);
    p.v_tree = static_cast<const __nv_bfloat16 *>(v_tree);
    p.k_pool = static_cast<const unsigned char *>(cache->k_pool);
    p.v_pool = static_cast<const unsigned char *>(cache->v_pool);
    p.page_table = cache->page_table;
    p.seq_lens = cache->seq_lens;
    p.parent = tree->parent;
    p.anc = tree->anc_mask;
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.lse = lse_out;
    p.status = status_out;
    p.B = B; p.T = T; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.D = D;
    p.max_pages = cache->max_pages_per_seq;
    p.num_pages = cache->num_pages;
    p.shared_prefix_pages = cache->shared_prefix_len / kPage;
    p.scale = softmax_scale;
    p.scale_log2 = softmax_scale * 1.4426950408889634f;
    p.give_up = ctx->q4_give_up;
    p.flags = reinterpret_cast<int32_t *>(ws + w.flags);
    p.partial_ml = reinterpret_cast<float2 *>(ws + w.partial_ml);
    p.partial_o = reinterpret_cast<float *>(ws + w.partial_o);
    p.tasks = reinterpret_cast<ShareTask *>(ws + w.tasks);
    p.inv_G = (unsigned)((((uint64_t)1 << 32) + p.G - 1) / p.G);
    bool few;
    if (reader_status s = q4_attn_rows_faster(&ctx->q4_attr, p, ctx->n_sm, &few)) return s;
    if (reader_status s = (few ? launch_q4_attn_rows : launch_q4_attn_sm100)(&ctx->q4_attr, p, ctx->n_sm, (cudaStream_t)stream)) return s;
    return launch_status();
}

size_t reader_pages_workspace_bytes(int32_t num_pages, int32_t rows, int32_t max_pages_per_seq, int32_t n) {
    if (num_pages < 1 || num_pages > kMost || rows < 1 || max_pages_per_seq < 1 || n < 0 || n > kMost || (int64_t)n * max_pages_per_seq >= (int64_t)1 << 31) return 0;
    return pages_layout(num_pages, rows, max_pages_per_seq, n).total;
}

reader_status reader_pages_fork(reader_ctx *ctx, const reader_pages *pages, const int32_t *src, const int32_t *dst, int32_t n, void *workspace,
                                size_t workspace_bytes, int32_t *status_out, void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (n == 0) return READER_OK;
    if (reader_status st = check_pages(pages, false)) return st;
    if (n < 0 || !src || !dst || !status_out) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_requests(pages, n, workspace, workspace_bytes)) return st;
    if (reader_status st = check_device(ctx)) return st;
    const PagesView v = view(pages);
    launch_pages_fork(v, src, dst, n, carve(pages_layout(v.num_pages, v.rows, v.width, n), workspace), status_out, (cudaStream_t)stream);
    return launch_status();
}

reader_status reader_pages_reserve(reader_ctx *ctx, const reader_pages *pages, const int32_t *rows, const int32_t *tokens, int32_t n, void *workspace,
                                   size_t workspace_bytes, int32_t *status_out, void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (n == 0) return READER_OK;
    if (reader_status st = check_pages(pages, true)) return st;
    if (n < 0 || !rows || !tokens || !status_out) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_requests(pages, n, workspace, workspace_bytes)) return st;
    if (reader_status st = check_device(ctx)) return st;
    std::vector<PoolList> chunks;
    if (reader_status st = pool_chunks(pages->pools, pages->pools, pages->n_pools, chunks)) return st;
    const PagesView v = view(pages);
    launch_pages_reserve(v, rows, tokens, n, carve(pages_layout(v.num_pages, v.rows, v.width, n), workspace), chunks.data(), pages->n_pools, pages->page_bytes,
                         status_out, (cudaStream_t)stream);
    return launch_status();
}

reader_status reader_pages_free(reader_ctx *ctx, const reader_pages *pages, const int32_t *rows, const int32_t *keep, int32_t n, int32_t *status_out,
                                void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (n == 0) return READER_OK;
    if (reader_status st = check_pages(pages, false)) return st;
    if (n < 0 || !rows || !status_out) return READER_ERR_INVALID_ARG;
    if (n > kMost) return READER_ERR_UNSUPPORTED;
    if (reader_status st = check_device(ctx)) return st;
    launch_pages_free(view(pages), rows, keep, n, status_out, (cudaStream_t)stream);
    return launch_status();
}

reader_status reader_pages_compact(reader_ctx *ctx, const reader_pages *pages, int32_t *n_used_out, void *workspace, size_t workspace_bytes, void *stream) {
    return reader_pages_compact_map(ctx, pages, n_used_out, nullptr, workspace, workspace_bytes, stream);
}

reader_status reader_pages_compact_map(reader_ctx *ctx, const reader_pages *pages, int32_t *n_used_out, int32_t *new_ids_out, void *workspace,
                                       size_t workspace_bytes, void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_pages(pages, true)) return st;
    if (!n_used_out) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_requests(pages, 0, workspace, workspace_bytes)) return st;
    if (reader_status st = check_device(ctx)) return st;
    std::vector<PoolList> chunks;
    if (reader_status st = pool_chunks(pages->pools, pages->pools, pages->n_pools, chunks)) return st;
    PagesView v = view(pages);
    v.new_ids = new_ids_out;
    launch_pages_compact(v, n_used_out, carve(pages_layout(v.num_pages, v.rows, v.width, 0), workspace), chunks.data(), pages->n_pools, pages->page_bytes,
                         ctx->n_sm, (cudaStream_t)stream);
    return launch_status();
}

reader_status reader_pages_copy(reader_ctx *ctx, const void *const *from_pools, int32_t from_pages, void *const *to_pools, int32_t to_pages,
                                int32_t n_pools, size_t page_bytes, const int32_t *from_ids, const int32_t *to_ids, int32_t n, int32_t *status_out,
                                void *stream) {
    if (!ctx) return READER_ERR_INVALID_ARG;
    if (n == 0) return READER_OK;
    if (!from_pools || !to_pools || from_pages < 0 || to_pages < 0 || n_pools < 1 || page_bytes == 0 || page_bytes % 16 != 0 || n < 0 || !from_ids ||
        !to_ids || !status_out)
        return READER_ERR_INVALID_ARG;
    if (page_bytes >= (size_t)1 << 31 || n > kMost) return READER_ERR_UNSUPPORTED;
    for (int i = 0; i < n_pools; ++i)
        if (!from_pools[i] || !to_pools[i] || !aligned16(from_pools[i]) || !aligned16(to_pools[i])) return READER_ERR_INVALID_ARG;
    if (reader_status st = check_device(ctx)) return st;
    std::vector<PoolList> chunks;
    if (reader_status st = pool_chunks(from_pools, to_pools, n_pools, chunks)) return st;
    launch_pages_copy(chunks.data(), n_pools, page_bytes, from_pages, to_pages, from_ids, to_ids, n, status_out, (cudaStream_t)stream);
    return launch_status();
}

}  // extern "C"

/*
 * reader_verify.h -- C ABI of the batched tree-verification step of READER-style lossless
 * speculative decoding, implemented as hand-written CUDA for sm_100a (NVIDIA B200).
 *
 * One decoding step of the method (Algorithm 1: the Verify call and the cache maintenance that
 * follows it) hands a draft tree per sequence to the target model, which scores every node in one
 * pass (Sec. 3.2), keeps the longest root path the model agrees with (Algorithm 5; Appendix C,
 * invariants 1-3) and appends the accepted entries to the KV cache without gaps (Sec. 4.3,
 * Algorithm 4).  This library is the attention, acceptance and cache part of that step:
 *
 *     reader_tree_encode   parent array  ->  per-node ancestor bitmask           (Sec. 3.2 mask)
 *     reader_verify_attn   tree-masked attention over paged cache + tree K/V     (Sec. 3.2)
 *     reader_accept        target argmax + longest consistent root path          (Algorithm 5)
 *     reader_kv_commit     accepted K/V rows -> cache tail, seq_lens += n_acc    (Algorithm 4)
 *   and, beside these: reader_sample_targets (the sampling policies of Appendix C in place of the
 *   argmax), reader_verify_prepare / reader_verify_attn_prepared (the per-step part of the attention call
 *   done once for all layers), reader_accept_commit (acceptance and commit in one launch), reader_kv_commit_layers (all
 *   layers of a model in one launch), reader_kv_rearrange
 *   (Algorithm 4 on the paper's padded cache layout), reader_verify_attn_padded /
 *   reader_padded_append / reader_padded_rearrange (the padded cache of Sec. 4.3 run as a cache, to be
 *   measured against the paged one), reader_accept_noalloc;
 *   and what comes before it: reader_prompt_append (head norms, position rotation and cache write of a prompt),
 *   reader_prompt_attn (its causal attention over the paged cache) and reader_tree_rotate (the same norms and rotation
 *   for draft nodes);
 *   and the cache itself: held in 4 bits, reader_q4_store / reader_q4_load / reader_q4_commit and reader_q4_verify_attn (the attention
 *   over it, draft trees and single tokens); its pages, reader_pages_fork / reader_pages_reserve / reader_pages_free / reader_pages_compact
 *   (reader_pages_compact_map) / reader_pages_copy.
 *
 * Conventions common to every call
 *   - Every pointer named below is a DEVICE pointer owned by the caller unless it says "host".
 *     The library allocates no device memory; scratch comes from the caller's workspace.
 *   - `stream` is a cudaStream_t passed as void*.  Calls only enqueue work on it: none of them
 *     synchronises or reads device data on the host.
 *   - Tensors are dense, row-major, last index fastest.  bf16 tensors are raw 16-bit patterns.
 *     Pointers to bf16/f32/u64 tensors must be 16-byte aligned.
 *   - Errors have two channels.  (1) The return value reports what the host can check (null or
 *     misaligned pointers, unsupported shapes, workspace too small, a CUDA launch error); on
 *     such an error nothing has been launched.  (2) `status_out[b]` (device, one word per
 *     sequence) reports what only the data can tell: a malformed parent array, a page id
 *     outside the pool, a length beyond the page table.  A sequence with a non-zero status gets
 *     defined outputs (attention rows and lse zero; n_acc 0, path -1, bonus -1; nothing
 *     committed) and does not disturb the others.  No kernel traps, asserts or waits unbounded.
 *   - A context is bound to one device and is not thread-safe: it caches the TMA descriptors of the
 *     tensors it saw last, so calls on one context come from one host thread at a time (use one
 *     context per thread or serialise).  Calls on different contexts are independent.
 *   - An empty batch (batch = 0) is legal everywhere: the call returns READER_OK, launches nothing
 *     and looks at no tensor pointer.
 *   - Tree convention: node 0 is the root = the last token already chosen by the target model
 *     (its K/V is part of the tree tensors, not yet of the cache); parent[0] = -1 and
 *     0 <= parent[j] < j.  At most READER_MAX_NODES nodes.
 */
#ifndef READER_VERIFY_H
#define READER_VERIFY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define READER_MAX_NODES 128
#define READER_PAGE_SIZE 64
#define READER_NOALLOC_MAX_ROWS 4096 /* batch * n_nodes limit of reader_accept_noalloc */

typedef struct reader_ctx reader_ctx; /* opaque: device id, SM count, driver entry points */

typedef enum {
    READER_OK = 0,
    READER_ERR_INVALID_ARG = 1, /* null/misaligned pointer, size out of range */
    READER_ERR_BAD_TREE = 2,    /* status word: parent array breaks the tree convention */
    READER_ERR_CAPACITY = 3,    /* status word: length beyond the page table / commit has no room */
    READER_ERR_WORKSPACE = 4,   /* workspace smaller than reader_workspace_bytes() */
    READER_ERR_UNSUPPORTED = 5, /* shape the kernels are not built for */
    READER_ERR_TIMEOUT = 6,     /* status word: a bounded device-side wait gave up */
    READER_ERR_CUDA = 7,        /* a CUDA runtime/driver call failed */
    READER_ERR_BAD_PAGE = 8,    /* status word: page-table entry outside [0, num_pages) */
    READER_ERR_TOO_LARGE = 9    /* more rows than reader_accept_noalloc's built-in scratch holds */
} reader_status;

/*
 * One layer's paged KV cache (Sec. 4.3: per-sample cache without internal padding).
 *   k_pool, v_pool   bf16 [num_pages][n_kv_heads][page_size][head_dim]
 *   page_table       i32  [batch][max_pages_per_seq]; entry p of row b is the pool page that
 *                    holds logical positions p*page_size .. p*page_size+page_size-1 of sequence b
 *   seq_lens         i32  [batch] committed tokens per sequence; read by reader_verify_attn,
 *                    updated by reader_kv_commit
 *   shared_prefix_len  tokens (multiple of page_size, 0 = none) whose pages are the same pool
 *                    pages in every row of page_table (stored once); commits never write there
 * page_size must be READER_PAGE_SIZE; head_dim 64 or 128.
 */
typedef struct {
    void *k_pool;
    void *v_pool;
    int32_t num_pages, page_size, n_kv_heads, head_dim;
    const int32_t *page_table;
    int32_t max_pages_per_seq;
    int32_t *seq_lens;
    int32_t shared_prefix_len;
} reader_kv_cache;

/*
 * The draft trees of one step (Sec. 3.2; built by the drafting side of Algorithm 1).
 *   parent     i32 [batch][n_nodes]
 *   anc_mask   u64 [batch][n_nodes][2]  bit i of the 128-bit word of node j is set iff node i is
 *              j itself or an ancestor of j (from reader_tree_encode); NULL = encode internally
 */
typedef struct {
    int32_t batch, n_nodes;
    const int32_t *parent;
    const uint64_t *anc_mask;
} reader_tree;

/* Creates a context for CUDA device `device` (host call; may initialise the CUDA context).
 * *out is host memory owned by the library until reader_destroy.  READER_ERR_UNSUPPORTED when the
 * device is not of compute capability 10.x or the tensor-core attention kernel cannot be set up on it
 * (no tensor-map encoder in the driver, too little shared memory): the library never serves calls
 * from a slower path on its own. */
reader_status reader_create(reader_ctx **out, int device);
void reader_destroy(reader_ctx *ctx);
const char *reader_status_string(reader_status s);

/* Chooses the attention kernel: 0 = automatic (the tensor-core kernel, as a single launch for calls with
 * few units and as preparation + attention + combine otherwise; the CUDA-core kernel only for the shapes
 * the former is not built for: a GQA group that does not divide 128, a non-positive scale), 1 = always
 * the CUDA-core kernel, 2 = the tensor-core kernel on the three-launch path or READER_ERR_UNSUPPORTED,
 * 3 = the tensor-core kernel as a single launch or READER_ERR_UNSUPPORTED (batch * n_kv_heads * M tiles
 * must fit the GPU in one wave).  All compute Sec. 3.2's attention; this is a testing aid. Host call. */
reader_status reader_set_attn_kernel(reader_ctx *ctx, int32_t which);

/* Chooses how reader_verify_attn divides its work among thread blocks: 0 = automatic, 1 = always equal
 * ranges of the flattened tile list (best balance), 2 = the aligned partition whenever a prefix is
 * shared (every KV stream cut at the same relative positions, so that the sequences sharing a prefix
 * walk it in step and a prefix larger than the L2 cache is fetched from HBM once; automatic above 48 MB
 * of shared K and V).  Results do not depend on the choice beyond rounding; this is a testing and
 * measuring aid.  Host call. */
reader_status reader_set_partition(reader_ctx *ctx, int32_t which);

/* Profiling aid (host call): when both are non-NULL cudaEvent_t handles, the next calls of
 * reader_verify_attn (and of its prepared and padded forms) record `start` on the stream right before the main attention kernel and
 * `stop` right after it (the preparation and combine kernels lie outside).  NULL, NULL turns it off. */
reader_status reader_set_timing_events(reader_ctx *ctx, void *start, void *stop);

/* The same for reader_accept and reader_accept_commit called with logits: the events bracket the argmax
 * kernel (the acceptance walk that follows lies outside).  NULL, NULL turns it off. */
reader_status reader_set_accept_timing_events(reader_ctx *ctx, void *start, void *stop);

/* Bytes of device scratch that reader_verify_attn / reader_accept need for at most `max_batch`
 * sequences of at most `max_nodes` nodes.  Host call, no CUDA work.  Returns 0 on bad arguments. */
size_t reader_workspace_bytes(const reader_ctx *ctx, int32_t max_batch, int32_t max_nodes,
                              int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim);

/*
 * Sec. 3.2 decoding mask.  For every sequence b and node j writes the 128-bit ancestor-or-self
 * set anc_mask_out[b][j][0..1] and level_out[b][j] = number of nodes on the path root..j (nullable).
 * status_out[b] = READER_ERR_BAD_TREE when parent[b] breaks the tree convention (its masks are
 * then zero).  1 <= n_nodes <= READER_MAX_NODES.
 */
reader_status reader_tree_encode(reader_ctx *ctx, const int32_t *parent, int32_t batch, int32_t n_nodes,
                                 uint64_t *anc_mask_out, int32_t *level_out, int32_t *status_out,
                                 void *stream);

/*
 * Sec. 3.2 verification attention.  For sequence b, node j and query head h (KV head h / G,
 * G = n_q_heads / n_kv_heads) the query q[b][j][h] attends, with scores scaled by
 * softmax_scale, to the committed keys 0 .. seq_lens[b]-1 of the paged cache and to the tree
 * keys k_tree[b][i] of the nodes i that are j or an ancestor of j.
 *   q, out          bf16 [batch][n_nodes][n_q_heads][head_dim]
 *   k_tree, v_tree  bf16 [batch][n_nodes][n_kv_heads][head_dim]
 *   lse_out         f32  [batch][n_nodes][n_q_heads], natural log of the softmax denominator; nullable
 *   workspace       at least reader_workspace_bytes(...) bytes, 256-byte aligned; contents are
 *                   scratch, calls that share it must not overlap on the GPU
 *   status_out      i32 [batch]
 * Arithmetic: bf16 inputs, fp32 accumulation and softmax, probabilities rounded to bf16 before the
 * value product where tensor cores are used, bf16 (nearest-even) output.
 */
reader_status reader_verify_attn(reader_ctx *ctx, const void *q, int32_t n_q_heads,
                                 const void *k_tree, const void *v_tree,
                                 const reader_kv_cache *cache, const reader_tree *tree,
                                 float softmax_scale, void *out, float *lse_out,
                                 void *workspace, size_t workspace_bytes, int32_t *status_out,
                                 void *stream);

/*
 * Algorithm 5 (the comparison with the base model's choice) with the greedy policy of Appendix C.  If `logits` (f32
 * [batch][n_nodes][vocab]) is given, target_ids[b][j] is first set to the lowest index of the
 * row maximum (a NaN never wins; a NaN in slot 0 counts as -inf); otherwise target_ids is read
 * as given (any policy's per-node choice, e.g. a sampler driven by coupled uniforms).
 * A node is accepted when it is the root or its parent is accepted and
 * node_tokens[node] == target_ids[parent].  Returns the longest accepted root path with at most
 * max_path nodes (lowest end node among equals; equal sibling tokens are all followed):
 *   path_out   i32 [batch][max_path] node ids from the root, padded with -1
 *   n_acc_out  i32 [batch] nodes on the path, root counted (>= 1 for a valid tree)
 *   bonus_out  i32 [batch] target_ids at the end node: the token to emit after the path
 * The tokens appended to the output this step are node_tokens[path[1..n_acc-1]] then bonus.
 * workspace: as for reader_verify_attn (used only when logits is given).
 */
reader_status reader_accept(reader_ctx *ctx, const reader_tree *tree, const int32_t *node_tokens,
                            const float *logits, int32_t vocab, int32_t *target_ids,
                            int32_t max_path, int32_t *path_out, int32_t *n_acc_out,
                            int32_t *bonus_out, void *workspace, size_t workspace_bytes,
                            int32_t *status_out, void *stream);

/*
 * Appendix C, randomized decoding: the per-node target of a sampling policy, x* = F(P, U_t), for
 * use as `target_ids` of reader_accept(logits = NULL).  F is temperature sampling through the
 * inverse CDF.  One uniform serves one output position: every node of tree level lv (root = 1)
 * uses uniforms[b][lv - 1], and the caller passes the same uniforms the plain (non-speculative) run
 * would use for those positions -- that coupling is what makes the decoded text identical.
 *   logits      f32 [batch][n_nodes][vocab], 16-byte aligned
 *   uniforms    f32 [batch][n_nodes], values in [0, 1) (clamped into it)
 *   temperature > 0
 *   top_k       0 = no filtering; k >= 1 keeps only the logits that are at least the k-th largest of
 *               their row (NaN counts as -inf; logits equal to that value are all kept)
 *   top_p       >= 1 = no filtering; 0 < p < 1 keeps, of what top_k left, the smallest set of highest
 *               logits whose weight reaches the share p (logits equal to the last admitted one are
 *               admitted with it)
 *   target_ids  i32 [batch][n_nodes] out
 * The CDF is integer arithmetic (fp32 weights from a fixed fused-multiply-add polynomial for
 * 2^x, truncated to 40 fractional bits; exact 64-bit sums; threshold (S * trunc(u 2^24)) >> 24;
 * first token whose inclusive prefix sum exceeds it), so the result does not depend on how the
 * sum is parallelised.  NaN and -inf logits are never drawn; a row without any weight gives 0.
 * vocab <= 2 Mi.  No workspace.
 */
reader_status reader_sample_targets(reader_ctx *ctx, const reader_tree *tree, const float *logits, int32_t vocab,
                                    const float *uniforms, float temperature, int32_t top_k, float top_p,
                                    int32_t *target_ids, void *stream);

/*
 * Sec. 4.3 / Algorithm 4 in per-step form.  For k < n_acc[b] the K/V rows of node path[b][k]
 * (all KV heads) are copied to logical position seq_lens[b] + k of sequence b, i.e. pool slot
 * page_table[b][(L+k)/page_size]*page_size + (L+k)%page_size, which is also written to
 * slots_out[b][k] (i32 [batch][max_path], -1 padded).  If update_seq_lens != 0, seq_lens[b] +=
 * n_acc[b] afterwards (pass 0 for all but the last layer that shares seq_lens).  A sequence
 * whose page table cannot hold the new positions, or that would write below
 * shared_prefix_len, gets READER_ERR_CAPACITY and is left untouched.
 */
reader_status reader_kv_commit(reader_ctx *ctx, reader_kv_cache *cache, const void *k_tree,
                               const void *v_tree, int32_t batch, int32_t n_nodes,
                               const int32_t *path, const int32_t *n_acc, int32_t max_path,
                               int32_t update_seq_lens, int32_t *slots_out, int32_t *status_out,
                               void *stream);

/*
 * reader_accept followed by reader_kv_commit for one layer, with the acceptance walk and the commit
 * in a single launch (Algorithm 5, then Sec. 4.3 / Algorithm 4 in per-step form): one dependent
 * launch fewer per decoding step.  Arguments and results are those of the two calls: status_out is
 * reader_accept's status word, commit_status_out reader_kv_commit's; path_out and n_acc_out are both
 * outputs of the walk and what is committed.
 */
reader_status reader_accept_commit(reader_ctx *ctx, const reader_tree *tree, const int32_t *node_tokens,
                                   const float *logits, int32_t vocab, int32_t *target_ids, int32_t max_path,
                                   reader_kv_cache *cache, const void *k_tree, const void *v_tree,
                                   int32_t update_seq_lens, int32_t *path_out, int32_t *n_acc_out,
                                   int32_t *bonus_out, int32_t *slots_out, void *workspace,
                                   size_t workspace_bytes, int32_t *status_out, int32_t *commit_status_out,
                                   void *stream);

/*
 * reader_kv_commit for every layer of a model in one launch (the accepted path is the same in all
 * layers; a 32-layer model would otherwise issue 32 small kernels per step).
 *   caches     HOST array [n_layers] of reader_kv_cache: each layer's own k_pool / v_pool; all layers
 *              must share page_table, seq_lens, num_pages, n_kv_heads, head_dim, max_pages_per_seq and
 *              shared_prefix_len (one block table for the whole model), else READER_ERR_INVALID_ARG
 *   k_trees, v_trees  HOST arrays [n_layers] of device pointers, bf16 [batch][n_nodes][n_kv_heads][head_dim]
 * slots_out, status_out and the seq_lens update are those of reader_kv_commit (the check has the
 * same outcome in every layer).  n_layers >= 1.
 */
reader_status reader_kv_commit_layers(reader_ctx *ctx, const reader_kv_cache *caches, const void *const *k_trees,
                                      const void *const *v_trees, int32_t n_layers, int32_t batch, int32_t n_nodes,
                                      const int32_t *path, const int32_t *n_acc, int32_t max_path,
                                      int32_t update_seq_lens, int32_t *slots_out, int32_t *status_out, void *stream);

/*
 * Sec. 4.3 / Algorithm 4 on the paper's own cache layout (not the paged cache of the calls above):
 * a rectangular batch cache whose per-sample rows hold real entries and internal padding.
 *   k, v         bf16 [batch][n_kv_heads][capacity][head_dim], compacted in place
 *   valid        u8   [batch][capacity]: non-zero marks a real entry (a mask; values are not tested
 *                for zero); rewritten to 1..10..0
 *   lengths_out  i32  [batch]: real entries per sample
 * Per sample the real entries move to the front in order (RemoveInternalZeroPadding +
 * TightConcatenate) and the vacated tail is zeroed.  head_dim a multiple of 8; k, v 16-byte aligned.
 */
reader_status reader_kv_rearrange(reader_ctx *ctx, void *k, void *v, int32_t batch, int32_t n_kv_heads,
                                  int32_t capacity, int32_t head_dim, uint8_t *valid, int32_t *lengths_out,
                                  void *stream);

/*
 * reader_verify_attn in two parts, for a model with several layers: all layers of a step see the same
 * trees, lengths and block table, so the checks, the masks and the work partition are made once
 * (reader_verify_prepare) and every layer then runs only its attention and combine kernels
 * (reader_verify_attn_prepared) -- one launch and several microseconds fewer per layer.
 *
 * reader_verify_prepare: cache->page_table / seq_lens / shapes and tree are read (k_pool, v_pool are
 * not); status_out (i32 [batch]) receives the status words of reader_verify_attn and stays in use by
 * the prepared calls.  The result lives in `workspace`.
 * reader_verify_attn_prepared: same arguments as reader_verify_attn, with this layer's q, k_tree,
 * v_tree, pools and out; workspace, batch, tree (parent and anc_mask pointers), n_q_heads and the
 * cache's page_table, seq_lens and shapes must be the ones given to the last reader_verify_prepare on
 * this context, else READER_ERR_INVALID_ARG.  Between the two nothing may change seq_lens, the page
 * table or the trees, and no other reader_verify_attn* call may use the workspace (reader_accept* may).
 * Rows of a rejected sequence are zeroed in every layer's out.  A bounded wait that gives up in one
 * layer marks all later layers of the step as well (READER_ERR_TIMEOUT in status_out, zero rows).
 */
reader_status reader_verify_prepare(reader_ctx *ctx, const reader_kv_cache *cache, const reader_tree *tree,
                                    int32_t n_q_heads, void *workspace, size_t workspace_bytes,
                                    int32_t *status_out, void *stream);
reader_status reader_verify_attn_prepared(reader_ctx *ctx, const void *q, int32_t n_q_heads, const void *k_tree,
                                          const void *v_tree, const reader_kv_cache *cache,
                                          const reader_tree *tree, float softmax_scale, void *out,
                                          float *lse_out, void *workspace, size_t workspace_bytes,
                                          void *stream);

/*
 * The padded batch cache of Sec. 4.3 as a cache in its own right: the layout the paper starts from,
 * kept here beside the paged cache so that the two designs can be run and measured against each
 * other.  Every sample owns one row of `capacity` positions; all rows are in use up to the common
 * length *extent; within a row real entries and padding alternate as the steps left them.
 *   k, v      bf16 [batch][n_kv_heads][capacity][head_dim]
 *   valid     u8   [batch][capacity]: non-zero marks a real entry; zero at and beyond *extent
 *             (the two calls that move *extent keep it so; the attention ignores bytes there anyway)
 *   extent    i32  [1] DEVICE scalar: rows at or beyond it are unused in every sample
 * Padding rows may hold anything (the calls below write zeros there, as the paper does): no
 * query ever sees them.
 */
typedef struct {
    void *k;
    void *v;
    uint8_t *valid;
    int32_t *extent;
    int32_t capacity, n_kv_heads, head_dim;
} reader_padded_cache;

/* Workspace for reader_verify_attn_padded: that of reader_workspace_bytes plus the packed mask. */
size_t reader_padded_workspace_bytes(const reader_ctx *ctx, int32_t max_batch, int32_t max_nodes,
                                     int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                     int32_t capacity);

/*
 * reader_verify_attn (Sec. 3.2) over a padded batch cache: node j of sample b attends over the
 * real entries of row b below *extent, in position order, and over the tree nodes on its root
 * path.  Arguments, outputs, kernels and error channels are those of reader_verify_attn; there is
 * no page table, and status_out[b] = READER_ERR_CAPACITY for every sample when *extent is outside
 * [0, capacity].  Every sample costs the common length, padding included: that is the overhead
 * Sec. 4.3 describes.  head_dim 64 or 128; k, v 16-byte aligned.
 */
reader_status reader_verify_attn_padded(reader_ctx *ctx, const void *q, int32_t n_q_heads, const void *k_tree,
                                        const void *v_tree, const reader_padded_cache *cache,
                                        const reader_tree *tree, float softmax_scale, void *out, float *lse_out,
                                        void *workspace, size_t workspace_bytes, int32_t *status_out,
                                        void *stream);

/*
 * One step's growth of a padded batch cache (Sec. 4.3: a long accepted span in one sample makes
 * every other sample pad up to the new maximum length).  The K/V rows of path[b][0 .. n_acc[b]-1]
 * are written at positions *extent .. *extent + n_acc[b] - 1 of row b and marked real; zero rows
 * marked padding fill row b up to *extent + max_b n_acc[b], which becomes the new *extent.
 *   k_tree, v_tree  bf16 [batch][n_nodes][n_kv_heads][head_dim];  path i32 [batch][max_path];
 *   n_acc i32 [batch] (the outputs of reader_accept)
 * All or nothing: when the new length exceeds capacity, an n_acc is outside [0, max_path] or a path
 * entry is not a node, every status_out[b] is READER_ERR_CAPACITY and nothing is changed.
 * head_dim a multiple of 8.
 */
reader_status reader_padded_append(reader_ctx *ctx, reader_padded_cache *cache, const void *k_tree,
                                   const void *v_tree, int32_t batch, int32_t n_nodes, const int32_t *path,
                                   const int32_t *n_acc, int32_t max_path, int32_t *status_out, void *stream);

/*
 * reader_kv_rearrange (Algorithm 4) on a reader_padded_cache, all `capacity` positions of it:
 * afterwards every row is compact, lengths_out[b] (i32 [batch]) holds its entries and *extent is
 * the longest of them.
 */
reader_status reader_padded_rearrange(reader_ctx *ctx, reader_padded_cache *cache, int32_t batch,
                                      int32_t *lengths_out, void *stream);

/*
 * reader_accept with target logits, for callers that cannot provide a workspace.  (The paper has
 * no counterpart: this exists only because of how the library is deployed.)  Think of a serving
 * process that gave all device memory to its own pool at start-up, or a decode loop that may not
 * make an allocating call between steps: neither can cudaMalloc the scratch reader_accept wants.
 * Here the per-block (maximum, index) pairs of the logits scan live in a 2 MiB array inside the
 * library's device image instead; every GPU that loads the library holds it until the process
 * exits.  Inputs, outputs and results are exactly those of reader_accept(logits != NULL).
 *   - batch * n_nodes must not exceed READER_NOALLOC_MAX_ROWS, else READER_ERR_TOO_LARGE is
 *     returned and nothing is launched.
 *   - The call allocates nothing.  Its first use on a device looks up the array's device address
 *     (once per device; the context's device must be current): make that first call before any
 *     stream capture begins.
 *   - All calls share the array and leave their pairs in it.  Nothing in it needs clearing, every
 *     slot read is written earlier in the same call; but calls that can overlap on the GPU (two
 *     streams, two host threads) race on it -- issue them on one stream or order them.
 *   - The events of reader_set_accept_timing_events are not recorded by this call.
 */
reader_status reader_accept_noalloc(reader_ctx *ctx, const reader_tree *tree, const int32_t *node_tokens,
                                    const float *logits, int32_t vocab, int32_t *target_ids,
                                    int32_t max_path, int32_t *path_out, int32_t *n_acc_out,
                                    int32_t *bonus_out, int32_t *status_out, void *stream);

/*
 * ---- From a prompt to a cache, from a projection to a tree --------------------------------------------------------
 * The calls above start from a cache that holds the prompt and from tree tensors that hold rotated keys.  The calls
 * below make both, in the same conventions:
 *   prompt, per layer:   reader_prompt_append -> reader_prompt_attn          (whole prompts, pieces of prompts, and
 *                                                                             single tokens without a draft)
 *   step, per layer:     reader_tree_rotate -> reader_verify_attn -> ...
 */

/*
 * New tokens of a batch, packed one sequence behind the other without padding.
 *   token_start   i32 [batch + 1]: rows token_start[b] .. token_start[b+1]-1 of the packed tensors belong to
 *                 sequence b (none when the two are equal); non-decreasing, within [0, total_tokens]
 *   total_tokens  rows of the packed tensors; rows outside every sequence are neither read nor written, so a
 *                 captured call may be given tensors larger than a step needs
 * Token i of sequence b stands at position seq_lens[b] + i: seq_lens counts the tokens committed before this call.
 * An array that breaks the convention gives READER_ERR_INVALID_ARG in every status word, and nothing else is written.
 */
typedef struct {
    int32_t batch, total_tokens;
    const int32_t *token_start;
} reader_prompt;

/*
 * What happens to a head of queries or keys x[0 .. head_dim-1] before it is used.
 *   q_weight, k_weight  bf16 [head_dim]: x := x * rsqrt(mean(x^2) + eps) * weight, per head; both NULL: no norm
 *   rope           f32 [max_positions][2][rot_dim / 2]: cosines, then sines, of each position's angles (any scaling of
 *                  the angles is the caller's); NULL: no rotation.  The first rot_dim elements of a head are rotated:
 *                  pair j is (j, j + rot_dim/2), or (2j, 2j + 1) if interleaved != 0:
 *                  (a, b) := (a cos - b sin, b cos + a sin)
 *   rot_dim        a multiple of 16, at most head_dim
 * fp32 arithmetic, one rounding (nearest even) to bf16 at the end.
 */
typedef struct {
    const void *q_weight, *k_weight;
    float eps;
    const float *rope;
    int32_t max_positions, rot_dim, interleaved;
} reader_rotation;

/*
 * A projection's output into the cache: queries and keys of the new tokens are normalised and rotated, keys and
 * values written to the pages of their positions seq_lens[b] + i, queries to q_out.  seq_lens is not changed (the last
 * layer's reader_prompt_attn advances it).
 *   q, k, v    bf16: head h of token t at q + t * q_stride + h * head_dim (strides in elements, multiples of 8): the
 *              parts of one fused tensor or tensors of their own
 *   q_out      bf16 [total_tokens][n_q_heads][head_dim]; may be q itself if q_stride = n_q_heads * head_dim
 *   status_out i32 [batch]: READER_ERR_CAPACITY when the page table or the rope table cannot hold the new positions
 *              or they begin below shared_prefix_len, READER_ERR_BAD_PAGE when a page that would be written is
 *              outside the pool: nothing of that sequence is written to the cache, its rows of q_out are zero
 * head_dim 64 or 128.  Sequences must not share a page that the call writes to.
 */
reader_status reader_prompt_append(reader_ctx *ctx, const void *q, const void *k, const void *v, int64_t q_stride,
                                   int64_t k_stride, int64_t v_stride, int32_t n_q_heads, reader_kv_cache *cache,
                                   const reader_prompt *prompt, const reader_rotation *rotation, void *q_out,
                                   int32_t *status_out, void *stream);

/*
 * The same for the nodes of draft trees: node j of sequence b stands at position seq_lens[b] + (nodes above it).
 *   q, k, v    as above, token row b * n_nodes + j
 *   q_out bf16 [batch][n_nodes][n_q_heads][head_dim], k_tree_out, v_tree_out bf16
 *              [batch][n_nodes][n_kv_heads][head_dim]: the q, k_tree, v_tree of reader_verify_attn and
 *              reader_kv_commit.  q_out (k_tree_out, v_tree_out) may be q (k, v) itself if that is dense.
 *   status_out i32 [batch]: READER_ERR_BAD_TREE; READER_ERR_CAPACITY when seq_lens[b] < 0 or the rope table is too
 *              short for the tree: that sequence's rows are zero
 * tree->anc_mask is not used.
 */
reader_status reader_tree_rotate(reader_ctx *ctx, const void *q, const void *k, const void *v, int64_t q_stride,
                                 int64_t k_stride, int64_t v_stride, int32_t n_q_heads, int32_t n_kv_heads,
                                 int32_t head_dim, const reader_tree *tree, const int32_t *seq_lens,
                                 const reader_rotation *rotation, void *q_out, void *k_tree_out, void *v_tree_out,
                                 int32_t *status_out, void *stream);

/* Bytes of device scratch that reader_prompt_attn needs, whatever the batch.  Host call, no CUDA work; 0 on bad
 * arguments. */
size_t reader_prompt_workspace_bytes(const reader_ctx *ctx, int32_t head_dim);

/*
 * Causal attention of the new tokens over the cache, which already holds their own keys and values (from
 * reader_prompt_append): token i of sequence b attends to the positions 0 .. seq_lens[b] + i.  With seq_lens[b] = 0 it
 * is a whole prompt, otherwise the next piece of one, with a single token plain decoding; a call may mix them.
 *   q, out     bf16 [total_tokens][n_q_heads][head_dim]; out may be q
 *   lse_out    f32 [total_tokens][n_q_heads], natural log of the softmax denominator; nullable
 *   update_seq_lens  non-zero: seq_lens[b] += new tokens afterwards (pass 0 for all but the last layer)
 *   workspace  at least reader_prompt_workspace_bytes(...) bytes, 256-byte aligned; contents are scratch, calls that
 *              share it must not overlap on the GPU
 *   status_out i32 [batch]: READER_ERR_CAPACITY, READER_ERR_BAD_PAGE, READER_ERR_TIMEOUT: that sequence's rows of out and
 *              lse_out are zero and its length is not advanced.  (After READER_ERR_TIMEOUT rows may also hold their values,
 *              and a later call with the same workspace may report the same event once more.)
 * READER_ERR_UNSUPPORTED unless: softmax_scale > 0 and at most 2e38; n_q_heads a multiple of n_kv_heads, at most 128 times it;
 * batch at most 32768; num_pages * n_kv_heads * 64 and max_pages_per_seq * 64 below 2^31; and, with g = 128 / (n_q_heads /
 * n_kv_heads) rounded down, (total_tokens / (2 g) + batch) * n_kv_heads * (max_pages_per_seq / 2 + 3) below 2^31.
 * How a call is divided is chosen on the host from batch, total_tokens and max_pages_per_seq, not from the lengths: a page
 * table or a captured call's tensors much larger than a step needs cost time (one token on 511: 10 or 19 us; one token on
 * 30000 in a call captured for 4096: 241 us instead of 32), and never results.  A shared prefix is read for each sequence.
 * What the cache holds at positions a token does not see has no influence on its row,
 * infinities and NaN included.
 * Arithmetic: bf16 inputs, fp32 accumulation and softmax, probabilities rounded to bf16 before the value product, bf16
 * (nearest-even) output.
 */
reader_status reader_prompt_attn(reader_ctx *ctx, const void *q, int32_t n_q_heads, reader_kv_cache *cache,
                                 const reader_prompt *prompt, float softmax_scale, int32_t update_seq_lens, void *out,
                                 float *lse_out, void *workspace, size_t workspace_bytes, int32_t *status_out,
                                 void *stream);

/* Testing aid (host call): thread block `cta` of each following reader_prompt_attn call on this context acts, once its work
 * is done, as one that gave up a bounded wait (READER_ERR_TIMEOUT); no wait runs out.  -1 turns it off. */
reader_status reader_set_prompt_give_up(reader_ctx *ctx, int32_t cta);

/*
 * ---- A cache in 4 bits ---------------------------------------------------------------------------------------------
 * The calls below keep a layer's keys and values in 4.5 bits an element instead of 16: 3.55 times the tokens in the same memory,
 * and as much less to read for each token.  In the same conventions:
 *   prompt, per layer:   reader_prompt_append -> reader_prompt_attn on a bf16 cache (one for all layers will do), then
 *                        reader_q4_store; a prompt that comes in pieces: reader_q4_load first
 *   step:                reader_tree_rotate -> reader_q4_verify_attn per layer -> reader_accept -> reader_q4_commit
 * A cache in 4 bits is a reader_kv_cache whose
 *   k_pool, v_pool   u8 [num_pages][n_kv_heads][36 * head_dim]: 64 positions of one head, numbers and scales
 * (csrc/q4_format.cuh has the places of the bits; these calls are the only ones that write or read them).
 *
 * 16 consecutive elements of a head share a scale s = (1 + m/8) 2^(e-18), m = 0..7, e = 0..31 (m < 7 if e = 31): the smallest with 7.5 s >=
 * their largest magnitude.  An element x is held as the whole number nearest x / s (ties to even), from -7 to 7, and stands for
 * that number of scales: within s / 2 of x, and exact in bf16.  Magnitudes above 107520 are held as the largest number; 16
 * elements with an infinity or a NaN among them all read as NaN.
 */

/*
 * Positions first[b] .. last[b] - 1 of every sequence from bf16 caches to 4-bit ones, layer by layer (none if first[b] >= last[b]).
 *   from, to     HOST arrays [n_layers]: from[i] in bf16, to[i] in 4 bits.  All of `from` share page_table, num_pages, n_kv_heads,
 *                head_dim and max_pages_per_seq, and so do all of `to` (and shared_prefix_len), else READER_ERR_INVALID_ARG; the two
 *                page tables may differ, heads and head_dim may not.  seq_lens are neither read nor changed and may be NULL.
 *   first, last  i32 [batch]
 *   status_out   i32 [batch]: READER_ERR_CAPACITY when first[b] < 0, first[b] < shared_prefix_len of `to` or a page table is too
 *                short, READER_ERR_BAD_PAGE when a page of either is outside its pool: nothing of that sequence is written
 * Positions outside the range keep what they hold.  Sequences must not share a page that the call writes to.  head_dim 64 or 128, at most
 * 2^30 sequences.
 */
reader_status reader_q4_store(reader_ctx *ctx, const reader_kv_cache *from, const reader_kv_cache *to, int32_t n_layers, int32_t batch,
                              const int32_t *first, const int32_t *last, int32_t *status_out, void *stream);

/* The other way: from[i] in 4 bits, to[i] in bf16; what the numbers stand for, exactly. */
reader_status reader_q4_load(reader_ctx *ctx, const reader_kv_cache *from, const reader_kv_cache *to, int32_t n_layers, int32_t batch,
                             const int32_t *first, const int32_t *last, int32_t *status_out, void *stream);

/* reader_kv_commit_layers into 4-bit caches (n_layers = 1: reader_kv_commit). */
reader_status reader_q4_commit(reader_ctx *ctx, const reader_kv_cache *caches, const void *const *k_trees, const void *const *v_trees,
                               int32_t n_layers, int32_t batch, int32_t n_nodes, const int32_t *path, const int32_t *n_acc,
                               int32_t max_path, int32_t update_seq_lens, int32_t *slots_out, int32_t *status_out, void *stream);

/* Bytes of device scratch that reader_q4_verify_attn needs, whatever the batch.  Host call, no CUDA work; 0 on bad arguments. */
size_t reader_q4_workspace_bytes(const reader_ctx *ctx, int32_t head_dim);

/*
 * reader_verify_attn over a cache in 4 bits: the committed keys and values are what the numbers stand for, those of the tree are
 * bf16 as ever.  A tree of one node is plain decoding.  Arguments, outputs and status words are those of reader_verify_attn, except
 *   workspace  at least reader_q4_workspace_bytes(...) bytes, 256-byte aligned; contents are scratch, calls that share it must
 *              not overlap on the GPU
 *   status_out READER_ERR_TIMEOUT besides (rows of that sequence may also hold their values)
 * READER_ERR_UNSUPPORTED unless: softmax_scale > 0 and at most 2e38; n_q_heads a multiple of n_kv_heads, at most 4096
 * times it; batch at most 65536; and batch *
 * n_kv_heads * (n_nodes * n_q_heads / n_kv_heads / 16 + 1) * (max_pages_per_seq + 4) below 2^31.
 * Small calls run as one launch, which goes by the page table's width: a token on 511 positions (32 query and 8 KV heads of 128) takes 7 to
 * 9 us, 13 behind a table of more than 191 pages; eight of them 8 us, 18 behind more than 95.
 * Bytes at positions that are not committed have no influence, whatever they are.  A row that sees nothing (an anc_mask without the
 * node itself, on an empty cache) is zero, its lse -inf.  Infinite or NaN values of a node reach the rows that see it, and no others; where
 * an infinite one's weight is 0 in fp32, as infinity or as NaN.
 * Arithmetic: fp32 accumulation and softmax (an exponent, in log2 units, to 2^-23 of the row's largest scaled score), probabilities
 * rounded to bf16 before the value product, bf16 (nearest-even) output.
 */
reader_status reader_q4_verify_attn(reader_ctx *ctx, const void *q, int32_t n_q_heads, const void *k_tree, const void *v_tree,
                                    const reader_kv_cache *cache, const reader_tree *tree, float softmax_scale, void *out,
                                    float *lse_out, void *workspace, size_t workspace_bytes, int32_t *status_out, void *stream);

/* Testing aid (host call): a share of the following reader_q4_verify_attn calls on this context acts as one whose bounded wait
 * ran out (READER_ERR_TIMEOUT); no wait runs out.  -1 turns it off. */
reader_status reader_set_q4_give_up(reader_ctx *ctx, int32_t worker);

/*
 * ---- The pages of a cache ------------------------------------------------------------------------------------------
 * Which page of the pools holds what is the caller's affair in the calls above: they follow page_table.  The calls below look
 * after the table on the device, without a host that waits for lengths, for caches of either kind.
 *   refs         i32 [num_pages]: how many entries of the page table name a page; 0 = the page is free.  The caller sets it up
 *                (all zero for an empty cache); pages that are not to be handed out get a count of their own (a compaction moves
 *                them as it moves others: reader_pages_compact_map tells where to)
 *   page_table   i32 [rows][max_pages_per_seq], -1 = no page (as for reader_kv_cache: one table for all layers of a model)
 *   seq_lens     i32 [rows]
 *   pools        HOST array [n_pools] of device pointers, 16-byte aligned: every pool whose pages the table names (keys and
 *                values of all layers), each num_pages * page_bytes bytes; page_bytes is a multiple of 16
 * Row numbers, counts and lengths live on the device; requests come as arrays [n], answers as status_out[n].  A request with a
 * status other than READER_OK changes nothing, unless it says so, and does not disturb the others.
 * Free pages are handed out lowest number first, in the order of the requests: the same inputs give the same pages.
 * Pages that a call takes out of the table are free for the next call.
 * READER_ERR_UNSUPPORTED: more than 2^30 pages or requests, pages of 2^31 bytes or more, rows of 2^31 positions or more.
 */
typedef struct {
    int32_t *refs;
    int32_t num_pages;
    int32_t *page_table;
    int32_t rows, max_pages_per_seq;
    int32_t *seq_lens;
    void *const *pools;
    int32_t n_pools;
    size_t page_bytes;
} reader_pages;

/* Bytes of device scratch that reader_pages_fork, reader_pages_reserve (of at most n requests) and reader_pages_compact need.
 * Host call, no CUDA work; 0 on bad arguments. */
size_t reader_pages_workspace_bytes(int32_t num_pages, int32_t rows, int32_t max_pages_per_seq, int32_t n);

/*
 * Row dst[i] becomes what row src[i] is: its length, and the pages of its positions, which both rows name from now on (no data
 * are copied).  The pages that row dst[i] named are released.  All at once: every source is read before any row is written, so rows
 * may be permuted (a beam search's reordering), one source may have many destinations, and src[i] = dst[i] is allowed.
 *   workspace   256-byte aligned; contents are scratch, calls that share it must not overlap on the GPU
 *   status_out  READER_ERR_INVALID_ARG: a row outside the table, or a dst that an earlier request names; READER_ERR_CAPACITY: a length
 *               outside [0, max_pages_per_seq * 64]; READER_ERR_BAD_PAGE: a page of the source's positions outside the pool
 * pools are not looked at.  n * max_pages_per_seq < 2^31, else READER_ERR_UNSUPPORTED (here and in reader_pages_reserve).
 */
reader_status reader_pages_fork(reader_ctx *ctx, const reader_pages *pages, const int32_t *src, const int32_t *dst, int32_t n,
                                void *workspace, size_t workspace_bytes, int32_t *status_out, void *stream);

/*
 * Makes positions seq_lens[r] .. seq_lens[r] + tokens[i] - 1 of row r = rows[i] the row's own to write: entries without a page get a
 * free one, entries whose page other entries name too get a free one in its place, and where such a page holds positions
 * below seq_lens[r] its data are copied, in all pools.  Whether a page is shared goes by refs before the call: two rows that share a
 * page and are both among the requests get a page each, and the shared one is released.
 *   status_out  READER_ERR_INVALID_ARG: a row outside the table or named by an earlier request, tokens[i] < 0; READER_ERR_BAD_PAGE
 *               (tokens[i] > 0): an entry outside the pool among those to write to, or no page where positions are committed;
 *               READER_ERR_CAPACITY: the row is too short for the new length, or too few pages are free: requests are served in
 *               order, and from the first that does not find enough on none that needs a page is
 * workspace as for reader_pages_fork.
 */
reader_status reader_pages_reserve(reader_ctx *ctx, const reader_pages *pages, const int32_t *rows, const int32_t *tokens, int32_t n,
                                   void *workspace, size_t workspace_bytes, int32_t *status_out, void *stream);

/*
 * Row rows[i] keeps its first keep[i] tokens (keep NULL: none): entries behind their pages are released and become -1, and the
 * length is lowered to keep[i] if it is larger.  A row may be named more than once (the lowest of the keeps counts).
 *   status_out  READER_ERR_INVALID_ARG: a row outside the table, keep[i] < 0; READER_ERR_BAD_PAGE: an entry outside the pool was among
 *               those that became -1
 * pools are not looked at.
 */
reader_status reader_pages_free(reader_ctx *ctx, const reader_pages *pages, const int32_t *rows, const int32_t *keep, int32_t n,
                                int32_t *status_out, void *stream);

/*
 * Moves the pages in use to the front of the pools: with n of them, those numbered n and above move, in ascending order, to the
 * free numbers below n, in ascending order; page_table and refs follow, the data of all pools move.  As few pages move as can.
 * Pages with a count of the caller's own move like the others, and so do those that another table over the same pools names:
 * who keeps numbers anywhere but in page_table needs reader_pages_compact_map.
 *   n_used_out  i32 [1]: pages in use; pages from that number on are free afterwards
 * workspace as for reader_pages_fork (any n).
 */
reader_status reader_pages_compact(reader_ctx *ctx, const reader_pages *pages, int32_t *n_used_out, void *workspace,
                                   size_t workspace_bytes, void *stream);

/* reader_pages_compact that tells where pages went.
 *   new_ids_out  i32 [num_pages] (NULL: not told): each page's new number, its own if it stays, -1 if it was free */
reader_status reader_pages_compact_map(reader_ctx *ctx, const reader_pages *pages, int32_t *n_used_out, int32_t *new_ids_out,
                                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Copies page from_ids[i] of from_pools[j] to page to_ids[i] of to_pools[j], for all i < n and j < n_pools: within pools or to others
 * (a page saved aside, a pool that grows).  HOST arrays of device pointers, 16-byte aligned; page_bytes a multiple of 16.
 * No page may be written twice, nor written and read, in one call.
 *   status_out  i32 [n]: READER_ERR_BAD_PAGE where an id is outside [0, from_pages) or [0, to_pages): nothing is copied
 */
reader_status reader_pages_copy(reader_ctx *ctx, const void *const *from_pools, int32_t from_pages, void *const *to_pools,
                                int32_t to_pages, int32_t n_pools, size_t page_bytes, const int32_t *from_ids, const int32_t *to_ids,
                                int32_t n, int32_t *status_out, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* READER_VERIFY_H */

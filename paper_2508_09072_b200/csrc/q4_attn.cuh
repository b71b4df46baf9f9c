// Parameter block and launchers of the attention over a 4-bit cache.
#pragma once
#include "common.cuh"

namespace reader {

constexpr int kQ4FewRows = 16;          // query rows of a KV head up to which the few-rows kernels are faster
// Rows of the shares of a thread block's workers and of its own two, at most (few-rows kernels).
constexpr int kQ4ShareRows = 512;   // (a block of the many-rows kernel: two shares of 256 rows)
constexpr int kQ4MaxBatch = 1 << 16;
constexpr int kQ4MaxGroup = 1 << 12;   // (128 nodes: 128 G^2 < 2^32, as the division by G wants it)

struct ShareTask {   // a unit that the thread blocks block0 .. block1 have shares of
    int b, h, rt, rows, block0, block1;   // block0 < 0: none
};

struct Q4AttnParams {
    const __nv_bfloat16 *q, *k_tree, *v_tree;
    const unsigned char *k_pool, *v_pool;
    const int32_t *page_table, *seq_lens, *parent;
    const uint64_t *anc;       // nullable: [B][T][2]
    __nv_bfloat16 *out;
    float *lse;                // nullable
    int32_t *status;
    int B, T, Hq, Hkv, G, D;
    int max_pages, num_pages, shared_prefix_pages;
    float scale_log2, scale;
    int give_up;               // worker that reports a wait that ran out (testing aid); -1: none
    // workspace
    int32_t *counters;         // [thread blocks] arrivals at the unit that a block begins and others go on with
    int32_t *flags;            // [2 * thread blocks] what is wrong with a block's shares
    float2 *partial_ml;        // [shares][rows] largest score, sum: of workers, behind them of blocks
    float *partial_o;          // [shares][rows][D]
    ShareTask *tasks;          // [thread blocks] the unit that a block begins and others go on with (many-rows kernel)
    int n_rt;                  // units of a KV head
    unsigned inv_G;            // 2^32 / G, rounded up
    int n_ctas;                // thread blocks (list form)
    int split;                 // thread blocks of a unit (alone)
};

// Which kernels have their attributes set.
struct Q4AttrSet {
    bool rows[4], sm100[2];
};
// Few query rows of a KV head (q4_attn_rows.cu), many (q4_attn_sm100.cu).
reader_status launch_q4_attn_rows(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, cudaStream_t st);
reader_status launch_q4_attn_sm100(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, cudaStream_t st);
// Zeroes the counters and the status words in front of a kernel that adds to them.
void launch_q4_attn_zero(const Q4AttnParams &p, int n_sm, cudaStream_t st);

}  // namespace reader

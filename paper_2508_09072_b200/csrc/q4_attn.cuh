// Parameter block and launchers of the attention over a 4-bit cache.
#pragma once
#include "common.cuh"

namespace reader {

// Query rows of a KV head up to which the few-rows kernels are faster: 32 sequences on 1024-4096, 16 rows 51 against 73 us, 32 rows 81 against 74.
constexpr int kQ4FewRows = 16;
constexpr int kQ4ShareRows = 512;      // rows of a thread block's shares: two of 256, or two of each worker's 8 or 16, at most
constexpr int kQ4Ranges = 16;          // ranges of a thread block, at most
constexpr int kQ4MaxBatch = 1 << 16;
constexpr int kQ4MaxGroup = 1 << 12;   // (128 nodes: 128 G^2 < 2^32, as the division by G wants it)

// A unit that several ranges of the work list (workers of the few-rows kernel, thread blocks of the many-rows one) have shares of.
struct ShareTask {
    int b, h, rt, rows, first, last;   // the ranges first .. last; first < 0: none
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
    int32_t *flags;            // [2 * ranges] what is wrong with a range's shares: of the unit it goes on with, of the unit it begins
    float2 *partial_ml;        // [2 * ranges][rows] largest score, sum
    float *partial_o;          // [2 * ranges][rows of D elements, in the kernel's own order]
    ShareTask *tasks;          // [ranges] the unit that a range begins and others go on with
    int n_rt;                  // units of a KV head
    unsigned inv_G;            // 2^32 / G, rounded up
    int n_ctas;                // thread blocks (list form)
    int split;                 // thread blocks of a unit (alone)
};

// Which kernels have their attributes set, and what was asked about them then.
constexpr int kQ4MaxCluster = 16;
struct Q4RowsKernels {
    bool set;
    int16_t clusters[kQ4MaxCluster + 1];   // of so many thread blocks that the GPU holds at a time
};
struct Q4AttrSet {
    Q4RowsKernels rows[4];   // head_dim 64, 128 (2); 8, 16 rows (1)
    bool sm100[2];
};
// Few query rows of a KV head (q4_attn_rows.cu), many (q4_attn_sm100.cu).  The former, too, for some small calls
// with more rows, in their form of one launch: 32 rows and 8 heads on 512 positions 9 against 15 us, 4 x 80 rows and 2 heads 12 against 18, 256 rows on 1400
// 21 against 26; but 8 x 128 rows on 1000, half a GPU full, 27 against 21, and they stay with the latter.
reader_status q4_attn_rows_faster(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, bool *yes);
reader_status launch_q4_attn_rows(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, cudaStream_t st);
reader_status launch_q4_attn_sm100(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, cudaStream_t st);
// The status words before a kernel raises some.
void launch_q4_attn_status(const Q4AttnParams &p, cudaStream_t st);

}  // namespace reader

// Parameter block and launchers of the attention over a 4-bit cache.
#pragma once
#include "common.cuh"

namespace reader {

// Workers (warps) of a thread block of the few-rows kernels, and rows of all of an SM's workers together, at most.
constexpr int kQ4MaxWorkers = 16, kQ4WorkerRows = 192;
constexpr int kQ4MaxBatch = 1 << 16;

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
    int32_t *counters;         // [4 * workers]: arrivals of a group's shares, of a unit's groups
    int32_t *flags;            // [2 * workers] what is wrong with a share
    float2 *partial_ml;        // [2 * workers][rows] largest score, sum
    float *partial_o;          // [2 * workers][rows][D]
    int n_ctas;                // thread blocks (list form)
    int split;                 // thread blocks of a unit (alone)
};

// Which kernels have their attributes set.
struct Q4AttrSet {
    bool rows[4];
};
reader_status launch_q4_attn_rows(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, cudaStream_t st);

}  // namespace reader

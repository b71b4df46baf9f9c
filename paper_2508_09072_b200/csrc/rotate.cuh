// Parameter block of the norm-and-rotation kernels (reader_prompt_append, reader_tree_rotate).
#pragma once
#include "common.cuh"

namespace reader {

struct RotateParams {
    const __nv_bfloat16 *q, *k, *v;            // token row i at base + i * stride (elements)
    int64_t q_stride, k_stride, v_stride;
    const __nv_bfloat16 *q_weight, *k_weight;  // both null: no norm
    const float *rope;                         // [max_positions][2][rot / 2]; null: no rotation
    float eps;
    int max_positions, rot, interleaved;
    int B, Hq, Hkv, D;
    const int32_t *seq_lens;
    __nv_bfloat16 *q_out, *k_out, *v_out;      // k_out, v_out: the pools, or the tree tensors
    int32_t *status;
    int share;                                 // warps that share a token's heads
    // prompt
    int tokens;                                // rows of the packed tensors
    const int32_t *token_start;                // [B + 1]
    const int32_t *page_table;
    int max_pages, num_pages, shared_prefix_len;
    // tree
    int T;
    const int32_t *parent;
};

void launch_prompt_append(RotateParams p, int n_sm, cudaStream_t st);
void launch_tree_rotate(RotateParams p, int n_sm, cudaStream_t st);

}  // namespace reader

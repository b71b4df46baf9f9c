// Launchers of the 4-bit cache's kernels outside the attention.
#pragma once
#include "common.cuh"

namespace reader {

// Pools (or tree tensors) of up to kQ4LayersPerLaunch layers, passed to the kernels by value.
constexpr int kQ4LayersPerLaunch = 32;
struct Q4Layers {
    const void *k_from[kQ4LayersPerLaunch], *v_from[kQ4LayersPerLaunch];
    void *k_to[kQ4LayersPerLaunch], *v_to[kQ4LayersPerLaunch];
};

struct Q4Convert {
    const int32_t *first, *last;           // [B] positions
    const int32_t *from_table, *to_table;  // [B][from_width], [B][to_width]
    int from_width, to_width, from_pages, to_pages;
    int shared_prefix_len;                 // of the destination
    int Hkv, D, B, layers;
    int per_seq;                           // thread blocks of a sequence
    bool whole;                            // the bf16 pools lie on 32-byte borders
    bool crowded;                          // a sequence may have more tiles than thread blocks
    int32_t *status;                       // null: not reported (layers behind the first launch)
};
void launch_q4_convert(bool store, Q4Convert p, const Q4Layers *chunks, int n_layers, int n_sm, cudaStream_t st);

struct Q4Commit {
    const int32_t *page_table;
    int max_pages, num_pages, shared_prefix_len;
    int32_t *seq_lens;
    const int32_t *path, *n_acc;
    int Hkv, D, B, T, max_path;
    int update;                            // seq_lens are advanced by the kernel itself (one layer only)
    int32_t *slots, *status;               // null: not reported
};
void launch_q4_commit(Q4Commit p, const Q4Layers *chunks, int n_layers, bool update_seq_lens, cudaStream_t st);

}  // namespace reader

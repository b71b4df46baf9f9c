// The 4-bit cache outside the attention: rows of a bf16 cache stored in 4 bits (reader_q4_store), their values loaded back
// (reader_q4_load), accepted tree rows committed (reader_q4_commit).
//
// Bound: bytes.  A block of 16 elements (32 bytes in bf16) belongs to one thread, from the loads to the numbers: the largest
// magnitude is found in its own registers, so nothing is exchanged and nothing is read twice.  Two neighbouring positions of a
// value tile share their words; the thread that has a block has both positions' (reading the word first where only one of them is
// written), so that no two threads of a launch write the same word.  Measured: 16 prompts of 100 to 4096 positions (8 heads, head_dim 128) stored in 40 us,
// loaded in 34, the copy bandwidth would allow 30.5; storing was bound by instructions until an element took six of them, and is on the
// border now.  Commits are latency: 16 sequences' paths of up to 8 nodes in 16 layers 5.3 us, in one layer of one sequence 2.5.
#include "q4_cache.cuh"
#include "q4_format.cuh"

namespace reader {
namespace {

constexpr int kThreads = 256;
constexpr int kCommitThreads = 512;   // (16 sequences, 16 layers, committed and loaded back: 12.3 us; 256: 13.8)

// A block of 16 elements in bf16: 32 bytes, by one instruction where the pools lie on such a border (two of 16 bytes each ask for every 32-byte sector
// twice), streamed past the caches' other users.
__device__ __forceinline__ void load_block(const uint4 *at, bool whole, uint4 (&x)[2]) {
    if (whole) {
        asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(x[0].x), "=r"(x[0].y), "=r"(x[0].z), "=r"(x[0].w), "=r"(x[1].x), "=r"(x[1].y), "=r"(x[1].z), "=r"(x[1].w)
                     : "l"(at));
    } else {
        x[0] = __ldcs(at);
        x[1] = __ldcs(at + 1);
    }
}
__device__ __forceinline__ void store_block(uint4 *at, bool whole, const uint4 &a, const uint4 &b) {
    if (whole) {
        asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x),
                     "r"(b.y), "r"(b.z), "r"(b.w)
                     : "memory");
    } else {
        __stcs(at, a);
        __stcs(at + 1, b);
    }
}

// What keeps the positions first .. last - 1 of sequence b from being converted.  Block-collective.
__device__ __forceinline__ int convert_status(const Q4Convert &p, int b, int first, int last) {
    if (last <= first) return READER_OK;
    const int64_t room = (int64_t)min(p.from_width, p.to_width) * kPage;
    if (first < 0 || first < p.shared_prefix_len || last > room) return READER_ERR_CAPACITY;
    bool bad = false;
    for (int i = first / kPage + threadIdx.x; i <= (last - 1) / kPage; i += kThreads) {
        const int a = p.from_table[(size_t)b * p.from_width + i], c = p.to_table[(size_t)b * p.to_width + i];
        bad |= a < 0 || a >= p.from_pages || c < 0 || c >= p.to_pages;
    }
    return __syncthreads_or(bad) ? READER_ERR_BAD_PAGE : READER_OK;
}

// One tile (page, head): rows lo .. hi - 1 of a bf16 tile of keys (values) to a 4-bit one.
template <int D>
__device__ __forceinline__ void store_tile(const __nv_bfloat16 *k, const __nv_bfloat16 *v, unsigned char *k4, unsigned char *v4, int lo, int hi, bool whole) {
    constexpr int kBlocks = D / q4::kBlock, kKeyTasks = kPage * kBlocks / kThreads, kPairs = kPage / 2 * kBlocks;
    const int tid = threadIdx.x;
    uint4 x[kKeyTasks][2], y[2][2];
#pragma unroll
    for (int i = 0; i < kKeyTasks; ++i) {
        const int task = i * kThreads + tid, r = task / kBlocks;
        if (r < lo || r >= hi) continue;
        load_block(reinterpret_cast<const uint4 *>(k) + task * 2, whole, x[i]);
    }
    const int t = tid / kBlocks, u = tid % kBlocks;   // value pair of this thread (128 of the 256 have none at head_dim 64)
    bool has[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        has[e] = tid < kPairs && 2 * t + e >= lo && 2 * t + e < hi;
        y[e][0] = y[e][1] = make_uint4(0, 0, 0, 0);
        if (!has[e]) continue;
        load_block(reinterpret_cast<const uint4 *>(v) + ((2 * t + e) * kBlocks + u) * 2, whole, y[e]);
    }
#pragma unroll
    for (int i = 0; i < kKeyTasks; ++i) {
        const int task = i * kThreads + tid, r = task / kBlocks;
        if (r >= lo && r < hi) q4::put_key_block<D>(k4, r, task % kBlocks, q4::quantise<true>(x[i][0], x[i][1]));
    }
    if (has[0] || has[1])
        q4::put_value_blocks<D>(v4, t, u, has[0], q4::quantise<false>(y[0][0], y[0][1]), has[1], q4::quantise<false>(y[1][0], y[1][1]));
}

// A position pair's words and codes of block u, and the pair's values from them.
template <int D>
__device__ __forceinline__ void read_pair(const unsigned char *v4, int t, int u, uint4 &words, int &codes) {
    constexpr int kChunkWords = D / 32;
    words = *reinterpret_cast<const uint4 *>(v4 + t * D + q4::v_chunk<D>(t, u * (4 / kChunkWords)) * kChunkWords * 4);
    codes = *reinterpret_cast<const uint16_t *>(v4 + q4::scales_at(D) + q4::v_scale_at<D>(2 * t, u));
}
template <int D>
__device__ __forceinline__ void write_pair(const uint4 &words, int codes, __nv_bfloat16 *v, int t, int u, const bool (&has)[2], bool whole) {
    constexpr int kBlocks = D / q4::kBlock;
    const uint32_t w[4] = {q4::plain_of(words.x), q4::plain_of(words.y), q4::plain_of(words.z), q4::plain_of(words.w)};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (!has[e]) continue;
        const float s = q4::scale_of((codes >> (8 * e)) & 255);
        const int sh = 16 * e;
        store_block(reinterpret_cast<uint4 *>(v) + ((2 * t + e) * kBlocks + u) * 2, whole,
                    q4::values_of(((w[0] >> sh) & 0xffffu) | (((w[1] >> sh) & 0xffffu) << 16), s),
                    q4::values_of(((w[2] >> sh) & 0xffffu) | (((w[3] >> sh) & 0xffffu) << 16), s));
    }
}

// The other way.
template <int D>
__device__ __forceinline__ void load_tile(const unsigned char *k4, const unsigned char *v4, __nv_bfloat16 *k, __nv_bfloat16 *v, int lo, int hi, bool whole) {
    constexpr int kBlocks = D / q4::kBlock, kKeyTasks = kPage * kBlocks / kThreads, kPairs = kPage / 2 * kBlocks;
    const int tid = threadIdx.x;
    uint2 kw[kKeyTasks];
    int kc[kKeyTasks];
#pragma unroll
    for (int i = 0; i < kKeyTasks; ++i) {
        const int task = i * kThreads + tid, r = task / kBlocks;
        if (r < lo || r >= hi) continue;
        kw[i] = *reinterpret_cast<const uint2 *>(k4 + task * 8);
        kc[i] = k4[q4::scales_at(D) + q4::k_scale_at<D>(r, task % kBlocks)];
    }
    const int t = tid / kBlocks, u = tid % kBlocks;
    const bool has[2] = {tid < kPairs && 2 * t >= lo && 2 * t < hi, tid < kPairs && 2 * t + 1 >= lo && 2 * t + 1 < hi};
    uint4 vw = make_uint4(0, 0, 0, 0);
    int vc = 0;
    if (has[0] || has[1]) read_pair<D>(v4, t, u, vw, vc);
#pragma unroll
    for (int i = 0; i < kKeyTasks; ++i) {
        const int task = i * kThreads + tid, r = task / kBlocks;
        if (r < lo || r >= hi) continue;
        const float s = q4::scale_of(kc[i]);
        store_block(reinterpret_cast<uint4 *>(k) + task * 2, whole, q4::values_of(q4::in_order(q4::plain_of(kw[i].x)), s),
                    q4::values_of(q4::in_order(q4::plain_of(kw[i].y)), s));
    }
    write_pair<D>(vw, vc, v, t, u, has, whole);
}

// A few rows of a tile, by a warp: a block of keys, or of a position pair of values, to a lane at a time.  Up to 16: of 16 sequences in 16 layers (8 heads, head_dim 128) 16
// positions are stored in 13.2 us and loaded in 10.2, by whole blocks in 14.0 and 11.2; 17 in 15.0 and 11.7, by whole blocks in 14.6 and 11.5.
constexpr int kFewPositions = 16;
template <int D, bool kStore>
__device__ __forceinline__ void few_rows(const void *k_from, const void *v_from, void *k_to, void *v_to, int lo, int hi, bool whole) {
    constexpr int kBlocks = D / q4::kBlock;
    const int t0 = lo / 2, keys = (hi - lo) * kBlocks, pairs = ((hi - 1) / 2 - t0 + 1) * kBlocks;
    for (int i = threadIdx.x & 31; i < keys + pairs; i += 32) {
        if (i < keys) {
            const int r = lo + i / kBlocks, u = i % kBlocks, task = r * kBlocks + u;
            if (kStore) {
                uint4 x[2];
                load_block(static_cast<const uint4 *>(k_from) + task * 2, whole, x);
                q4::put_key_block<D>(static_cast<unsigned char *>(k_to), r, u, q4::quantise<true>(x[0], x[1]));
            } else {
                const unsigned char *k4 = static_cast<const unsigned char *>(k_from);
                const uint2 w = *reinterpret_cast<const uint2 *>(k4 + task * 8);
                const float s = q4::scale_of(k4[q4::scales_at(D) + q4::k_scale_at<D>(r, u)]);
                store_block(static_cast<uint4 *>(k_to) + task * 2, whole, q4::values_of(q4::in_order(q4::plain_of(w.x)), s),
                            q4::values_of(q4::in_order(q4::plain_of(w.y)), s));
            }
        } else {
            const int t = t0 + (i - keys) / kBlocks, u = (i - keys) % kBlocks;
            const bool has[2] = {2 * t >= lo, 2 * t + 1 < hi};
            if (kStore) {
                uint4 y[2][2] = {};
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (has[e]) load_block(static_cast<const uint4 *>(v_from) + ((2 * t + e) * kBlocks + u) * 2, whole, y[e]);
                q4::put_value_blocks<D>(static_cast<unsigned char *>(v_to), t, u, has[0], q4::quantise<false>(y[0][0], y[0][1]), has[1],
                                        q4::quantise<false>(y[1][0], y[1][1]));
            } else {
                uint4 words;
                int codes;
                read_pair<D>(static_cast<const unsigned char *>(v_from), t, u, words, codes);
                write_pair<D>(words, codes, static_cast<__nv_bfloat16 *>(v_to), t, u, has, whole);
            }
        }
    }
}

// Blocks b * per_seq .. + per_seq - 1 walk the tiles (layer, page, head) of sequence b, heads fastest; a warp to a tile where a sequence
// may have more tiles than blocks and the range has few positions (8 of 16 sequences in 16 layers loaded in 7.1 us, by whole blocks in 10.4; one sequence's in one layer 3.1
// and 2.5).
template <int D, bool kStore>
__global__ void __launch_bounds__(kThreads) q4_convert_kernel(const Q4Convert p, const __grid_constant__ Q4Layers layers) {
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.x / p.per_seq, x = blockIdx.x - b * p.per_seq;
    const int first = p.first[b], last = p.last[b];
    const bool few = p.crowded && last > first && (unsigned)last - (unsigned)first <= kFewPositions;
    constexpr int kWarps = kThreads / 32;
    if (few && x > 0 && x * kWarps >= ((last - 1) / kPage - first / kPage + 1) * p.Hkv * p.layers) return;   // (the first block looks at everything)
    const int st = convert_status(p, b, first, last);
    if (x == 0 && threadIdx.x == 0 && p.status) p.status[b] = st;
    if (st != READER_OK || last <= first) return;
    const int page0 = first / kPage, n_pages = (last - 1) / kPage - page0 + 1;
    constexpr size_t kWide = (size_t)kPage * D * sizeof(__nv_bfloat16), kNarrow = q4::tile_bytes(D), kFrom = kStore ? kWide : kNarrow, kTo = kStore ? kNarrow : kWide;
    if (few) {
        for (int i = x * kWarps + (threadIdx.x >> 5); i < n_pages * p.Hkv * p.layers; i += p.per_seq * kWarps) {
            const int h = i % p.Hkv, j = i / p.Hkv, l = j / n_pages, page = page0 + j - l * n_pages;
            const size_t from = (size_t)p.from_table[(size_t)b * p.from_width + page] * p.Hkv + h, to = (size_t)p.to_table[(size_t)b * p.to_width + page] * p.Hkv + h;
            few_rows<D, kStore>(static_cast<const unsigned char *>(layers.k_from[l]) + from * kFrom, static_cast<const unsigned char *>(layers.v_from[l]) + from * kFrom,
                                static_cast<unsigned char *>(layers.k_to[l]) + to * kTo, static_cast<unsigned char *>(layers.v_to[l]) + to * kTo,
                                max(0, first - page * kPage), min(kPage, last - page * kPage), p.whole);
        }
        return;
    }
    // item (l, page, h) number x + k per_seq, by carrying (a division each time costs as much as an eighth of the tile)
    const int q = x / p.Hkv, dq = p.per_seq / p.Hkv, dh = p.per_seq - dq * p.Hkv, dl = dq / n_pages, dj = dq - dl * n_pages;
    int h = x - q * p.Hkv, l = q / n_pages, j = q - l * n_pages;
    while (l < p.layers) {
        const int page = page0 + j;
        const int lo = max(0, first - page * kPage), hi = min(kPage, last - page * kPage);
        const size_t from = (size_t)p.from_table[(size_t)b * p.from_width + page] * p.Hkv + h;
        const size_t to = (size_t)p.to_table[(size_t)b * p.to_width + page] * p.Hkv + h;
        const unsigned char *k = static_cast<const unsigned char *>(layers.k_from[l]) + from * kFrom, *v = static_cast<const unsigned char *>(layers.v_from[l]) + from * kFrom;
        unsigned char *k_to = static_cast<unsigned char *>(layers.k_to[l]) + to * kTo, *v_to = static_cast<unsigned char *>(layers.v_to[l]) + to * kTo;
        if (kStore) store_tile<D>(reinterpret_cast<const __nv_bfloat16 *>(k), reinterpret_cast<const __nv_bfloat16 *>(v), k_to, v_to, lo, hi, p.whole);
        else load_tile<D>(k, v, reinterpret_cast<__nv_bfloat16 *>(k_to), reinterpret_cast<__nv_bfloat16 *>(v_to), lo, hi, p.whole);
        h += dh;
        j += dj;
        l += dl;
        if (h >= p.Hkv) { h -= p.Hkv; ++j; }
        if (j >= n_pages) { j -= n_pages; ++l; }
    }
}

// Block (b, l) commits sequence b into layer l: the accepted nodes' rows to the positions seq_lens[b] + k.
template <int D>
__global__ void __launch_bounds__(kCommitThreads) q4_commit_kernel(const Q4Commit p, const __grid_constant__ Q4Layers layers) {
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kBlocks = D / q4::kBlock;
    const int b = blockIdx.x, l = blockIdx.y, tid = threadIdx.x;
    const int L = p.seq_lens[b], n = p.n_acc[b];
    const int32_t *table = p.page_table + (size_t)b * p.max_pages, *path = p.path + (size_t)b * p.max_path;
    int32_t *slots = p.slots && l == 0 ? p.slots + (size_t)b * p.max_path : nullptr;
    bool bad = n > 0 && (n > p.max_path || L < 0 || L < p.shared_prefix_len || (int64_t)L + n > (int64_t)p.max_pages * kPage);
    if (!bad)
        for (int k = tid; k < n; k += kCommitThreads) {
            const int page = table[(L + k) / kPage], node = path[k];
            bad |= page < 0 || page >= p.num_pages || node < 0 || node >= p.T;
        }
    bad = __syncthreads_or(bad);
    if (tid == 0 && p.status && l == 0) p.status[b] = bad ? READER_ERR_CAPACITY : READER_OK;
    if (slots)
        for (int k = tid; k < p.max_path; k += kCommitThreads)
            slots[k] = !bad && k < n ? table[(L + k) / kPage] * kPage + (L + k) % kPage : -1;
    if (bad || n <= 0) return;
    auto row = [&](const void *tree, int k, int h, int u) {
        return reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(tree) + (((size_t)b * p.T + path[k]) * p.Hkv + h) * D + u * q4::kBlock);
    };
    auto tile = [&](void *pool, int pos, int h) {
        return static_cast<unsigned char *>(pool) + ((size_t)table[pos / kPage] * p.Hkv + h) * q4::tile_bytes(D);
    };
    const int per_pos = p.Hkv * kBlocks, key_tasks = n * per_pos;
    const int pair0 = L / 2, value_tasks = ((L + n - 1) / 2 - pair0 + 1) * per_pos;
    for (int i = tid; i < key_tasks + value_tasks; i += kCommitThreads) {
        if (i < key_tasks) {
            const int k = i / per_pos, h = (i - k * per_pos) / kBlocks, u = i % kBlocks;
            const uint4 *src = row(layers.k_from[l], k, h, u);
            q4::put_key_block<D>(tile(layers.k_to[l], L + k, h), (L + k) % kPage, u, q4::quantise<true>(src[0], src[1]));
        } else {
            const int j = i - key_tasks, pair = j / per_pos, h = (j - pair * per_pos) / kBlocks, u = j % kBlocks;
            const int pos = 2 * (pair0 + pair);   // the pair's even position
            const bool has_even = pos >= L, has_odd = pos + 1 < L + n;
            const uint4 *even = row(layers.v_from[l], has_even ? pos - L : 0, h, u), *odd = row(layers.v_from[l], has_odd ? pos + 1 - L : 0, h, u);
            const uint4 x[4] = {even[0], even[1], odd[0], odd[1]};
            q4::put_value_blocks<D>(tile(layers.v_to[l], pos, h), (pos % kPage) / 2, u, has_even, q4::quantise<false>(x[0], x[1]), has_odd, q4::quantise<false>(x[2], x[3]));
        }
    }
    if (p.update) {   // the only block that reads this length
        __syncthreads();
        if (tid == 0) p.seq_lens[b] = L + n;
    }
}

__global__ void __launch_bounds__(kThreads) q4_advance_kernel(int32_t *__restrict__ seq_lens, const int32_t *__restrict__ n_acc,
                                                              const int32_t *__restrict__ status, int B) {
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.x * kThreads + threadIdx.x;
    if (b < B && status[b] == READER_OK && n_acc[b] > 0) seq_lens[b] += n_acc[b];
}

}  // namespace

void launch_q4_convert(bool store, Q4Convert p, const Q4Layers *chunks, int n_layers, int n_sm, cudaStream_t st) {
    // The lengths live on the device: as many thread blocks for a sequence as fill the GPU sixteen times over with all of them,
    // at most one per tile of the narrower table.
    const int32_t *status = p.status;
    for (int l0 = 0; l0 < n_layers; l0 += kQ4LayersPerLaunch) {
        p.layers = n_layers - l0 < kQ4LayersPerLaunch ? n_layers - l0 : kQ4LayersPerLaunch;
        const int64_t tiles = (int64_t)(p.from_width < p.to_width ? p.from_width : p.to_width) * p.Hkv * p.layers;
        const int64_t share = (16 * (int64_t)n_sm + p.B - 1) / p.B;
        p.per_seq = (int)(tiles < share ? tiles : share);
        p.crowded = tiles > share;
        p.status = l0 == 0 ? const_cast<int32_t *>(status) : nullptr;
        const Q4Layers &c = chunks[l0 / kQ4LayersPerLaunch];
        uintptr_t places = 0;
        for (int l = 0; l < p.layers; ++l)
            places |= store ? reinterpret_cast<uintptr_t>(c.k_from[l]) | reinterpret_cast<uintptr_t>(c.v_from[l])
                            : reinterpret_cast<uintptr_t>(c.k_to[l]) | reinterpret_cast<uintptr_t>(c.v_to[l]);
        p.whole = places % 32 == 0;
        auto kernel = p.D == 128 ? (store ? q4_convert_kernel<128, true> : q4_convert_kernel<128, false>)
                                 : (store ? q4_convert_kernel<64, true> : q4_convert_kernel<64, false>);
        launch_pdl(kernel, dim3((unsigned)(p.B * p.per_seq)), dim3(kThreads), 0, st, p, chunks[l0 / kQ4LayersPerLaunch]);
    }
}

void launch_q4_commit(Q4Commit p, const Q4Layers *chunks, int n_layers, bool update_seq_lens, cudaStream_t st) {
    int32_t *status = p.status, *slots = p.slots;
    p.update = update_seq_lens && n_layers == 1;
    for (int l0 = 0; l0 < n_layers; l0 += kQ4LayersPerLaunch) {
        const int layers = n_layers - l0 < kQ4LayersPerLaunch ? n_layers - l0 : kQ4LayersPerLaunch;
        p.status = l0 == 0 ? status : nullptr;
        p.slots = l0 == 0 ? slots : nullptr;
        launch_pdl(p.D == 128 ? q4_commit_kernel<128> : q4_commit_kernel<64>, dim3((unsigned)p.B, (unsigned)layers), dim3(kCommitThreads), 0, st, p,
                   chunks[l0 / kQ4LayersPerLaunch]);
    }
    if (update_seq_lens && n_layers > 1)
        launch_pdl(q4_advance_kernel, dim3((unsigned)((p.B + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, p.seq_lens, p.n_acc,
                   static_cast<const int32_t *>(status), p.B);
}

}  // namespace reader

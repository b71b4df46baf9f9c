// Tree-masked attention over a 4-bit cache for many query rows (reader_q4_verify_attn): draft trees, on the tcgen05 tensor cores.
//
// Bound: the tensor pipe and the exponentials, 2048 cycles each for 256 query rows and 128 keys; what 4 bits add is turning
// numbers into bf16 operands, 16384 of them for each, once for all rows that share them.  So a thread block (one per SM) has up to
// 256 rows of one KV head, two slots of 128, and four warps of it do nothing but unpack: a tile of 128 keys (two pages) becomes
// the rows of K, and its values the rows of V^T (position pairs are neighbours in the pages, so a pair of numbers is a
// pair of bf16 along the value product's inner axis as it stands), in the 128-byte swizzle of the matrix instructions.
//
//   warps 0-3, 4-7   softmax of slot 0 and 1: a thread per row.  Scores come from tensor memory; the maximum in use is raised when a
//                    score exceeds it by 2^8 (O is rescaled in tensor memory then); probabilities replace the scores as bf16 and are the
//                    value product's A operand from there.  At a unit's end they fetch the next one's queries, so that its first
//                    products run beside the results being written.
//   warps 8-11       unpack pages (and copy the tree's own keys and values) into the tiles
//   warp 12          brings pages into a ring by bulk copies
//   warp 13          issues the products: S = Q K^T, O += P V
//   warp 14          zero rows for sequences whose length cannot be
// A unit of more than 128 rows is wide: each slot has its own rows and both work on every tile.  A narrow one has up to 128 rows;
// the slots take the tiles in turns and their two results are merged at its end.
//
// Tensor memory: S of either slot (128 columns each; P over its first 64), O of either slot.  The products of a slot are issued by one
// thread and run in order, so S[i + 1] may be written over P[i] as soon as the value product that reads it has been issued.
//
// Work: a flat list of tiles cut into equal ranges, one per thread block, shares of units in several ranges merged by the block that
// comes last (q4_attn_common.cuh).  Bytes that are not committed never reach a product: their scores become -inf, and their values 0 or
// not multiplied at all (16-key slices behind the end).  Every wait is bounded: a block that gives up reports all its units.
#include <cuda.h>

#include "prompt_ptx.cuh"
#include "q4_attn_common.cuh"

namespace reader {
namespace {

using namespace q4;

constexpr int kThreads = 512;
constexpr int kSoftmaxThreads = 256;
constexpr int kUnpackWarp = 8, kLoadWarp = 12, kMmaWarp = 13, kRejectWarp = 14;
// Registers of a thread: softmax, unpacking, the rest; 128 (2 x 184 + 80 + 64) = 65536, what the block is launched with.
constexpr int kRegsSoftmax = 184, kRegsUnpack = 80, kRegsRest = 64;
constexpr int kTileKeys = 128;     // keys of a tile: two pages
constexpr int kUnitCost = 6;       // entries that stand for a unit's start and end
constexpr int kMinEntries = 8;     // of a range
constexpr int kRawSlots = 3;       // of the ring: keys or values of a tile's pages each
constexpr int kAhead = 8;          // units that a role may be ahead of another, at most (two tiles and a ring of one and a half)
constexpr uint32_t kTmemCols = 512, kTmemS = 0, kTmemO = 256;

template <int D>
struct Cfg {
    static constexpr int kPageBytes = tile_bytes(D);
    static constexpr int kHalves = D / 64;                    // 64-column blocks of a row of queries or keys
    static constexpr int kBlock = 128 * 128;                  // bytes of such a block, 128 rows
    static constexpr int kVPage = D * 128;                    // a page of V^T: D rows of 64 positions
    static constexpr int kQBytes = kHalves * kBlock;          // queries of a slot; keys of a tile
    static constexpr int kKBytes = kHalves * kBlock;
    static constexpr int kVBytes = 2 * kVPage;
    static constexpr int kOffQ = 0;
    static constexpr int kOffK = 2 * kQBytes;
    static constexpr int kOffV = kOffK + 2 * kKBytes;
    static constexpr int kOffRaw = kOffV + 2 * kVBytes;
    static constexpr int kRawBytes = 2 * kPageBytes;
    static constexpr int kOffParents = kOffRaw + kRawSlots * kRawBytes;   // kAhead / 2 trees
    static constexpr int kOffMl = kOffParents + kAhead / 2 * kMaxNodes;   // (m, l) of slot 1's rows, and of slot 0's
    static constexpr int kOffTable = kOffMl + 2 * 128 * 8;
    static constexpr int kOffBars = kOffTable + kPrefix * 8;
    static constexpr int kSmem = kOffBars + 512;
    static_assert(kSmem + 512 <= 227 * 1024, "shared memory");
};

struct ShareTask {   // a unit that other blocks have shares of
    int b, h, rt, rows, block0, block1;   // block0 < 0: none
};
struct Bars {
    uint64_t raw_full[kRawSlots], raw_empty[kRawSlots], k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t q_full, q_empty, s_full[2], p_full[2][2], o_full[2];
    uint32_t tmem_base;
    int32_t abort;
    int32_t raw_bad[kRawSlots];   // a page outside the pool among the slot's
    int32_t flags[kAhead];        // what is wrong with unit i mod kAhead
    int32_t poison[kAhead];       // its tree has infinities or NaN among the values
    int32_t last[2];
    int32_t warp_sum[kThreads / 32];
    ShareTask task[2];
};
static_assert(sizeof(Bars) <= 512, "barrier block");

// Bounded wait of a whole warp.  False, in every lane, when the block has given up.
__device__ __forceinline__ bool gone(volatile int32_t *abort_s) { return __any_sync(0xffffffffu, *abort_s != 0); }
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int32_t *abort_s) {
    bool ok = mbar_try_wait(bar, parity);
    if (__all_sync(0xffffffffu, ok)) return true;
    const uint64_t t0 = globaltimer_ns();
    while (true) {
        ok = ok || mbar_try_wait(bar, parity);
        if (__all_sync(0xffffffffu, ok)) return true;
        if (gone(abort_s)) return false;
        if (globaltimer_ns() - t0 > kWaitLimitNs) *abort_s = 1;
    }
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint16_t x;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(a));
    return x;
}
__device__ __forceinline__ void softmax_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory"); }

// A block's walk over its range: the units, and how their tiles are dealt out.
struct Walk {
    int w, w_end, seg;      // seg: units so far
    Unit u;
    int tiles, rows, visits;   // tiles here; rows of the unit; score products (both slots')
    bool wide, whole;
    __device__ __forceinline__ bool next(const Q4AttnParams &p, const List &l, const Seqs &s, int lane) {
        while (w < w_end) {
            u = unit_at(p, l, s, w, w_end, lane);
            w += u.entries;
            if (!u.any) continue;
            tiles = u.t1 - u.t0;
            rows = min(256, p.T * p.G - u.rt * 256);
            wide = u.weight == 2;
            visits = wide ? 2 * tiles : tiles;
            whole = u.t0 == 0 && u.t1 == u.ntiles;
            ++seg;
            return true;
        }
        return false;
    }
    __device__ __forceinline__ int tile_of(int visit) const { return wide ? visit >> 1 : visit; }
    // committed tiles of the sequence; the tree's tile comes behind them
    __device__ __forceinline__ int committed() const { return u.ntiles - 1; }
    __device__ __forceinline__ bool is_tree(int tile) const { return u.t0 + tile == committed(); }
    __device__ __forceinline__ int valid(const Q4AttnParams &p, int tile) const { return is_tree(tile) ? p.T : min(kTileKeys, u.L - (u.t0 + tile) * kTileKeys); }
};

// ---- unpacking, by 128 threads (`t` among them)
// A page of keys into rows row0 .. + 63 of a K tile.  Thread (w, g): word w of the positions 8 j + g (at head_dim 64, of half of the j).
template <int D>
__device__ __forceinline__ void unpack_keys(uint32_t raw, uint32_t tile, int row0, int t, uint32_t sixteen) {
    constexpr int kWords = D / 8, kPer = D / 64;   // words of a position; scale blocks of a quarter of it
    constexpr int kSplit = 128 / (8 * kWords);
    const int w = t % kWords, g = (t / kWords) & 7, u = w >> 1, j0 = t / (kWords * 8) * (8 / kSplit);
    // the codes of the positions 8 j + g: bytes kPer j + u mod kPer of 8 kPer
    const uint32_t at = raw + scales_at(D) + (g * 4 + u / kPer) * 8 * kPer + j0 * kPer;
    uint32_t codes[4] = {};
    if constexpr (D == 128) { const uint4 x = lds128(at); codes[0] = x.x; codes[1] = x.y; codes[2] = x.z; codes[3] = x.w; }
    else codes[0] = lds32(at);
    const uint32_t dst = tile + (w >> 3) * Cfg<D>::kBlock + (row0 + 8 * j0 + g) * 128 + (((w & 7) ^ g) << 4), src = raw + (8 * j0 + g) * (D / 2) + w * 4;
#pragma unroll
    for (int j = 0; j < 8 / kSplit; ++j) {
        const uint32_t word = lds32(src + j * 8 * (D / 2));
        const int byte = j * kPer;
        const uint32_t sel = (byte & 3) + (kPer == 2 ? (u & 1) : 0);
        const Scale2 s = scale2<false>(__byte_perm(codes[byte >> 2], 0, 0x4040 | sel | (sel << 8)));
        sts128(dst + j * 8 * 128, pair<0>(word, s, sixteen), pair<1>(word, s, sixteen), pair<2>(word, s, sixteen), pair<3>(word, s, sixteen));
    }
}
// A page of values into a page of V^T, `valid` of its positions committed (the others become 0).  64 threads: (q, z) = the positions 8 q .. + 7 of
// the elements z D/8 .. + D/8 - 1.
template <int D>
__device__ __forceinline__ void unpack_values(uint32_t raw, uint32_t page, int valid, int t, uint32_t sixteen) {
    constexpr int kWords = D / 32;
    const int q = t & 7, z = t >> 3;
    if (8 * q >= ((valid + 15) & ~15)) return;   // (behind the last slice that is multiplied)
    // The four position pairs 4 q + e, each lane's in an order that begins with e = q mod 4 (in one order for all, eight lanes would meet in
    // the same banks): k-th load e = (k + q) mod 4.
    uint32_t w[4][kWords], codes[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int e = (k + q) & 3, pr = 4 * q + e;
        const uint32_t at = raw + pr * D + v_chunk<D>(pr, z) * (D / 8);
        if constexpr (D == 128) { const uint4 x = lds128(at); w[k][0] = x.x; w[k][1] = x.y; w[k][2] = x.z; w[k][3] = x.w; }
        else { const uint2 x = lds64(at); w[k][0] = x.x; w[k][1] = x.y; }
        codes[k] = lds16(raw + scales_at(D) + ((((D == 128 ? z : z >> 1) * 4 + e) * 8 + q) * 2));
    }
    // back in order: turned by q mod 4
#pragma unroll
    for (int step = 1; step < 4; step <<= 1) {
        const bool turn = q & step;
#pragma unroll
        for (int y = 0; y <= kWords; ++y) {
            uint32_t a[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int from = (k - step) & 3;
                a[k] = y < kWords ? (turn ? w[from][y % kWords] : w[k][y % kWords]) : (turn ? codes[from] : codes[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (y < kWords) w[k][y % kWords] = a[k];
                else codes[k] = a[k];
            }
        }
    }
    Scale2 s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        s[e] = scale2<false>(__byte_perm(codes[e], 0, 0x4140));
        const int key = 8 * q + 2 * e;
        if (key >= valid) { s[e].s &= 0xffff0000u; s[e].m24 &= 0xffff0000u; }
        if (key + 1 >= valid) { s[e].s &= 0xffffu; s[e].m24 &= 0xffffu; }
    }
#pragma unroll
    for (int y = 0; y < kWords; ++y) {
        const int d0 = z * (D / 8) + 4 * y;
        auto row = [&](int i) { return page + (d0 + i) * 128 + ((q ^ ((d0 + i) & 7)) << 4); };
        sts128(row(0), pair<0>(w[0][y], s[0], sixteen), pair<0>(w[1][y], s[1], sixteen), pair<0>(w[2][y], s[2], sixteen), pair<0>(w[3][y], s[3], sixteen));
        sts128(row(1), pair<1>(w[0][y], s[0], sixteen), pair<1>(w[1][y], s[1], sixteen), pair<1>(w[2][y], s[2], sixteen), pair<1>(w[3][y], s[3], sixteen));
        sts128(row(2), pair<2>(w[0][y], s[0], sixteen), pair<2>(w[1][y], s[1], sixteen), pair<2>(w[2][y], s[2], sixteen), pair<2>(w[3][y], s[3], sixteen));
        sts128(row(3), pair<3>(w[0][y], s[0], sixteen), pair<3>(w[1][y], s[1], sixteen), pair<3>(w[2][y], s[2], sixteen), pair<3>(w[3][y], s[3], sixteen));
    }
}
// The tree's own keys as a K tile.
template <int D>
__device__ __forceinline__ void copy_tree_keys(const Q4AttnParams &p, int b, int h, uint32_t tile, int t) {
    constexpr int kChunks = D / 8;
#pragma unroll 4
    for (int i = t; i < p.T * kChunks; i += 128) {
        const int r = i / kChunks, w = i % kChunks;
        const uint4 x = *reinterpret_cast<const uint4 *>(p.k_tree + (((size_t)b * p.T + r) * p.Hkv + h) * D + w * 8);
        sts128(tile + (w >> 3) * Cfg<D>::kBlock + r * 128 + (((w & 7) ^ (r & 7)) << 4), x.x, x.y, x.z, x.w);
    }
}
// Its values as V^T: nodes 8 q .. + 7 of eight elements at a time.  Infinities and NaN become 0 (0 times them is NaN for the rows that do not see
// them); whether there were any.
template <int D>
__device__ __forceinline__ bool copy_tree_values(const Q4AttnParams &p, int b, int h, uint32_t tile, int t) {
    constexpr int kChunks = D / 8;
    const int groups = (p.T + 15) / 16 * 2;   // of eight nodes, up to the last slice's end
    bool dirty = false;
#pragma unroll 1
    for (int i = t; i < groups * kChunks; i += 128) {
        const int z = i % kChunks, q = i / kChunks;
        uint4 x[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            x[n] = make_uint4(0, 0, 0, 0);
            if (8 * q + n < p.T) x[n] = *reinterpret_cast<const uint4 *>(p.v_tree + (((size_t)b * p.T + 8 * q + n) * p.Hkv + h) * D + z * 8);
            dirty |= clean(x[n]);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            auto word = [&](int n) { return w == 0 ? x[n].x : w == 1 ? x[n].y : w == 2 ? x[n].z : x[n].w; };
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                const int d = z * 8 + 2 * w + odd;
                const uint32_t sel = odd ? 0x7632 : 0x5410;
                sts128(tile + (q >> 3) * Cfg<D>::kVPage + d * 128 + (((q & 7) ^ (d & 7)) << 4), __byte_perm(word(0), word(1), sel), __byte_perm(word(2), word(3), sel),
                       __byte_perm(word(4), word(5), sel), __byte_perm(word(6), word(7), sel));
            }
        }
    }
    return dirty;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) q4_attn_sm100_kernel(const __grid_constant__ Q4AttnParams p) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Bars *m = reinterpret_cast<Bars *>(smem + C::kOffBars);
    volatile int32_t *abort_s = &m->abort;
    auto bar = [&](const uint64_t *b) { return smem_u32(b); };
    if (tid == 0) {
        for (int i = 0; i < kRawSlots; ++i) {
            mbar_init(bar(&m->raw_full[i]), 1);
            mbar_init(bar(&m->raw_empty[i]), 4);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&m->k_full[i]), 4);
            mbar_init(bar(&m->k_empty[i]), 1);
            mbar_init(bar(&m->v_full[i]), 4);
            mbar_init(bar(&m->v_empty[i]), 1);
            mbar_init(bar(&m->s_full[i]), 1);
            mbar_init(bar(&m->p_full[i][0]), 128);
            mbar_init(bar(&m->p_full[i][1]), 128);
            mbar_init(bar(&m->o_full[i]), 1);
            m->task[i].block0 = -1;
            m->last[i] = 0;
        }
        mbar_init(bar(&m->q_full), kSoftmaxThreads);
        mbar_init(bar(&m->q_empty), 1);
        for (int i = 0; i < kAhead; ++i) m->flags[i] = m->poison[i] = 0;
        m->abort = (base & 1023u) ? 1 : 0;   // (the swizzled tiles want 1024-byte alignment; never seen otherwise, but checked)
        fence_mbar_init();
        fence_proxy_async();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&m->tmem_base), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = m->tmem_base;
    pdl_wait();
    pdl_launch_dependents();

    List list;
    list.cost = kUnitCost;
    list.pages = 2;
    list.weight = 2;
    const int rows_all = p.T * p.G;
    list.n_wide = rows_all / 256 + (rows_all % 256 > 128 ? 1 : 0);
    list.narrow = rows_all % 256 >= 1 && rows_all % 256 <= 128;
    list.tree_tiles = 1;
    Seqs seqs;
    make_list<kThreads / 32>(p, list, seqs, reinterpret_cast<int2 *>(smem + C::kOffTable), m->warp_sum);
    __syncthreads();
    list.per_block = 1;
    list.cut(max(1, min(p.n_ctas, list.W / kMinEntries)));
    Walk k;
    k.seg = -1;
    k.w = k.w_end = 0;
    if ((int)blockIdx.x < list.n_workers && list.W > 0) {
        k.w = list.begin(blockIdx.x);
        k.w_end = list.begin(blockIdx.x + 1);
    }

    if (warp >= 12) {
        regs_dec<kRegsRest>();
        if (warp == kLoadWarp) {
            // ------------------------------------------------------------------ pages
            const uint64_t policy = l2_policy_evict_first();
            const bool once = list.n_wide + list.narrow == 1;   // no other unit reads these pages
            int n = 0;   // slots of the ring so far
            while (!gone(abort_s) && k.next(p, list, seqs, lane)) {
                const int pages_end = min(k.u.npages, 2 * k.u.t1);
                int ids = 0, at = -32;
                for (int t = 0; t < k.tiles && !gone(abort_s); ++t) {
                    if (k.is_tree(t)) break;
                    const int page0 = 2 * (k.u.t0 + t);
                    if (page0 - at >= 32) {
                        at = page0;
                        ids = page0 + lane < pages_end ? p.page_table[(size_t)k.u.b * p.max_pages + page0 + lane] : 0;
                    }
                    const int id0 = __shfl_sync(0xffffffffu, ids, page0 - at), id1 = __shfl_sync(0xffffffffu, ids, page0 - at + 1);
                    const int count = min(2, pages_end - page0);
                    const bool ok0 = id0 >= 0 && id0 < p.num_pages, ok1 = count < 2 || (id1 >= 0 && id1 < p.num_pages);
                    const bool streamed = once && page0 >= p.shared_prefix_pages;
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const int s = n % kRawSlots;
                        if (!wait(bar(&m->raw_empty[s]), ((n / kRawSlots) & 1) ^ 1, abort_s)) break;
                        if (lane == 0) {
                            m->raw_bad[s] = !(ok0 && ok1);
                            const uint32_t full = bar(&m->raw_full[s]), dst = base + C::kOffRaw + s * C::kRawBytes;
                            const unsigned char *pool = kv ? p.v_pool : p.k_pool;
                            const int bytes = (ok0 ? C::kPageBytes : 0) + (count == 2 && ok1 ? C::kPageBytes : 0);
                            mbar_arrive_expect_tx(full, bytes);   // (a page outside the pool is not read; what the slot holds is never shown)
                            if (ok0) bulk_load(dst, pool + ((size_t)id0 * p.Hkv + k.u.h) * C::kPageBytes, C::kPageBytes, full, policy, streamed);
                            if (count == 2 && ok1) bulk_load(dst + C::kPageBytes, pool + ((size_t)id1 * p.Hkv + k.u.h) * C::kPageBytes, C::kPageBytes, full, policy, streamed);
                        }
                        __syncwarp();
                    }
                }
            }
            if (gone(abort_s)) {   // the block does not end under its own copies
                const uint64_t t0 = globaltimer_ns();
                for (int i = max(0, n - kRawSlots); i < n; ++i)
                    while (!mbar_try_wait(bar(&m->raw_full[i % kRawSlots]), (i / kRawSlots) & 1) && globaltimer_ns() - t0 < 20000000ull) {
                    }
            }
        } else if (warp == kMmaWarp) {
            // ------------------------------------------------------------------ products
            constexpr uint32_t kIdescQK = idesc_bf16_f32(128, kTileKeys, false, false), kIdescPV = idesc_bf16_f32(128, D, false, false);
            const uint64_t descQ = smem_desc_sw128(base + C::kOffQ, 16, 1024), descK = smem_desc_sw128(base + C::kOffK, 16, 1024);
            const uint64_t descV = smem_desc_sw128(base + C::kOffV, 16, 1024);
            int done = 0;                 // tiles of the units before
            uint32_t p_parity = 0;        // one bit per slot
            while (!gone(abort_s) && k.next(p, list, seqs, lane)) {
                wait(bar(&m->q_full), k.seg & 1, abort_s);
                auto score = [&](int v) {
                    const int slot = v & 1, t = k.tile_of(v), n = done + t, buf = n & 1;
                    wait(bar(&m->k_full[buf]), (n >> 1) & 1, abort_s);
                    tc_fence_after();
                    __syncwarp();
                    if (!gone(abort_s) && elect_one()) {
                        const uint64_t qd = descQ + (uint64_t)((k.wide ? slot * C::kQBytes : 0) >> 4), kd = descK + (uint64_t)((buf * C::kKBytes) >> 4);
#pragma unroll
                        for (int hf = 0; hf < C::kHalves; ++hf)
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                mma_bf16_ss(tmem + kTmemS + slot * 128, qd + (uint64_t)((hf * C::kBlock + kk * 32) >> 4), kd + (uint64_t)((hf * C::kBlock + kk * 32) >> 4),
                                            kIdescQK, (hf | kk) != 0);
                        mma_commit(bar(&m->s_full[slot]));
                        if (!k.wide || slot == 1) mma_commit(bar(&m->k_empty[buf]));
                        if (v == k.visits - 1) mma_commit(bar(&m->q_empty));
                    }
                    __syncwarp();
                };
                for (int v = 0; v < min(2, k.visits); ++v) score(v);
                for (int v = 0; v < k.visits; ++v) {
                    const int slot = v & 1, t = k.tile_of(v), n = done + t, buf = n & 1;
                    const int slices = (k.valid(p, t) + 15) >> 4;
                    const uint32_t tS = tmem + kTmemS + slot * 128, tO = tmem + kTmemO + slot * D;
                    wait(bar(&m->v_full[buf]), (n >> 1) & 1, abort_s);
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        wait(bar(&m->p_full[slot][half]), (p_parity >> slot) & 1, abort_s);
                        tc_fence_after();
                        __syncwarp();
                        if (!gone(abort_s) && elect_one()) {
                            const uint64_t vd = descV + (uint64_t)((buf * C::kVBytes + half * C::kVPage) >> 4);
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                if (half * 4 + kk < slices)
                                    mma_bf16_ts(tO, tS + (half * 4 + kk) * 8, vd + (uint64_t)((kk * 32) >> 4), kIdescPV, v >= 2 || half + kk != 0);
                            if (half == 1) {
                                if (!k.wide || slot == 1) mma_commit(bar(&m->v_empty[buf]));
                                if (v + 2 >= k.visits) mma_commit(bar(&m->o_full[slot]));
                            }
                        }
                        __syncwarp();
                    }
                    p_parity ^= 1u << slot;
                    if (v + 2 < k.visits) score(v + 2);
                }
                done += k.tiles;
            }
            if (gone(abort_s)) __nanosleep(1000000);   // products that are still under way end before their operands go away
        } else if (warp == kRejectWarp) {
            reject_lengths<D>(p, blockIdx.x, gridDim.x, lane);
        }
    } else if (warp >= kUnpackWarp) {
        // ------------------------------------------------------------------ unpacking
        regs_dec<kRegsUnpack>();
        const int t = tid - kUnpackWarp * 32;
        volatile uint32_t *word = reinterpret_cast<volatile uint32_t *>(smem + C::kOffMl);   // (an opaque constant: see pair())
        if (t == 0) *word = 0x41804180u;
        asm volatile("bar.sync 2, 128;" ::: "memory");
        const uint32_t sixteen = *word;
        asm volatile("bar.sync 2, 128;" ::: "memory");
        int n = 0, raw = 0, trees = 0;   // tiles, slots of the ring, trees so far
        while (!gone(abort_s) && k.next(p, list, seqs, lane)) {
            for (int i = 0; i < k.tiles && !gone(abort_s); ++i, ++n) {
                const int buf = n & 1;
                const uint32_t kt = base + C::kOffK + buf * C::kKBytes, vt = base + C::kOffV + buf * C::kVBytes;
                const bool tree = k.is_tree(i);
                const int valid = k.valid(p, i);
                // keys
                if (!wait(bar(&m->k_empty[buf]), ((n >> 1) & 1) ^ 1, abort_s)) break;
                if (tree) {
                    unsigned char *parents = smem + C::kOffParents + (trees & (kAhead / 2 - 1)) * kMaxNodes;
                    if (t < p.T) {
                        const int a = p.parent[(size_t)k.u.b * p.T + t];
                        parents[t] = (unsigned char)a;
                        if (!(t == 0 ? a == -1 : a >= 0 && a < t)) atomicOr(&m->flags[k.seg & (kAhead - 1)], kBadTree);
                    }
                    copy_tree_keys<D>(p, k.u.b, k.u.h, kt, t);
                    ++trees;
                } else {
                    const int s = raw % kRawSlots;
                    if (!wait(bar(&m->raw_full[s]), (raw / kRawSlots) & 1, abort_s)) break;
                    const uint32_t src = base + C::kOffRaw + s * C::kRawBytes;
                    if (m->raw_bad[s] && t == 0) atomicOr(&m->flags[k.seg & (kAhead - 1)], kBadPage);
                    unpack_keys<D>(src, kt, 0, t, sixteen);
                    if (valid > kPage) unpack_keys<D>(src + C::kPageBytes, kt, kPage, t, sixteen);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&m->raw_empty[s]));
                    ++raw;
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&m->k_full[buf]));
                // values
                if (!wait(bar(&m->v_empty[buf]), ((n >> 1) & 1) ^ 1, abort_s)) break;
                if (tree) {
                    if (copy_tree_values<D>(p, k.u.b, k.u.h, vt, t)) atomicOr(&m->poison[k.seg & (kAhead - 1)], 1);
                } else {
                    const int s = raw % kRawSlots;
                    if (!wait(bar(&m->raw_full[s]), (raw / kRawSlots) & 1, abort_s)) break;
                    const uint32_t src = base + C::kOffRaw + s * C::kRawBytes;
                    // a page to 64 threads
                    if (t < 64) unpack_values<D>(src, vt, min(valid, kPage), t, sixteen);
                    else if (valid > kPage) unpack_values<D>(src + C::kPageBytes, vt + C::kVPage, valid - kPage, t - 64, sixteen);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&m->raw_empty[s]));
                    ++raw;
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&m->v_full[buf]));
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax, results
        regs_inc<kRegsSoftmax>();
        const int slot = warp >> 2, row = tid & 127;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + kTmemS + slot * 128 + lane_base, tO = tmem + kTmemO + slot * D + lane_base;
        constexpr uint32_t kNegInf = 0xff800000u;
        float2 *ml_s = reinterpret_cast<float2 *>(smem + C::kOffMl);
        const float by = kRaiseBy / p.scale_log2;
        uint32_t s_parity = 0, o_parity[2] = {0, 0};
        int trees = 0;   // (both slots count all of them)

        // Queries of unit x: rows of this slot (wide) or this slot's half of the columns of all of them (narrow).
        auto load_queries = [&](const Walk &x) {
            const int r = x.u.rt * 256 + (x.wide ? slot * 128 : 0) + row;
            const bool live = r < p.T * p.G;
            const int j = live ? node_of(p, r) : 0, hq = x.u.h * p.G + (live ? r - j * p.G : 0);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (((size_t)x.u.b * p.T + j) * p.Hq + hq) * D);
            constexpr int kChunks = D / 8;
            const uint32_t dst = base + C::kOffQ + (x.wide ? slot * C::kQBytes : 0) + row * 128;
            const int c0 = x.wide ? 0 : slot * (kChunks / 2);
            auto part = [&](int c1) {
#pragma unroll
                for (int i = 0; i < kChunks / 2; ++i) {
                    const int ch = c1 + i;
                    const uint4 q = live ? src[ch] : make_uint4(0, 0, 0, 0);
                    sts128(dst + (ch >> 3) * C::kBlock + (((ch & 7) ^ (row & 7)) << 4), q.x, q.y, q.z, q.w);
                }
            };
            part(c0);
            if (x.wide) part(kChunks / 2);
            fence_proxy_async();
            mbar_arrive(bar(&m->q_full));
        };
        // (Given up or not, every thread goes through all units: the barriers among the softmax threads want that.)
        bool more = k.next(p, list, seqs, lane);
        if (more) load_queries(k);
        while (more) {
            const int grow = k.u.rt * 256 + (k.wide ? slot * 128 : 0) + row;   // among the head's rows
            const bool live = grow < p.T * p.G;
            const bool warp_live = __any_sync(0xffffffffu, live);
            const int node = live ? node_of(p, grow) : 0;
            // a row without a query never asks for a higher maximum
            float mx = live ? -INFINITY : INFINITY, l = 0.f;
            const bool has_tree = k.is_tree(k.tiles - 1);
            for (int v = slot; v < k.visits; v += 2) {
                const int t = k.tile_of(v);
                wait(bar(&m->s_full[slot]), s_parity, abort_s);
                s_parity ^= 1;
                tc_fence_after();
                if (warp_live) {
                    uint32_t s[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(s + c * 32));
                    tmem_wait_ld();
                    auto f = [&](int i) { return __uint_as_float(s[i]); };
                    if (k.is_tree(t)) {
                        uint64_t lo = 0, hi = 0;   // the nodes this row sees
                        if (live) {
                            if (p.anc) {
                                lo = p.anc[((size_t)k.u.b * p.T + node) * 2];
                                hi = p.anc[((size_t)k.u.b * p.T + node) * 2 + 1];
                            } else if (!(*(volatile int32_t *)&m->flags[k.seg & (kAhead - 1)] & kBadTree)) {
                                const unsigned char *parents = smem + C::kOffParents + (trees & (kAhead / 2 - 1)) * kMaxNodes;
                                for (int i = node; i != 255; i = parents[i]) {   // (strictly falling on a valid tree)
                                    if (i < 64) lo |= 1ull << i;
                                    else hi |= 1ull << (i - 64);
                                }
                            }
                        }
                        if (p.T < 64) lo &= (1ull << p.T) - 1;
                        if (p.T < 128) hi &= p.T <= 64 ? 0 : (1ull << (p.T - 64)) - 1;
#pragma unroll
                        for (int i = 0; i < 64; ++i) {
                            if (!((lo >> i) & 1)) s[i] = kNegInf;
                            if (!((hi >> i) & 1)) s[64 + i] = kNegInf;
                        }
                    } else {
                        const int valid = k.valid(p, t);
                        if (valid < kTileKeys) {
#pragma unroll
                            for (int i = 0; i < kTileKeys; ++i)
                                if (i >= valid) s[i] = kNegInf;
                        }
                    }
                    float tops[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float a = max3(f(c * 32), f(c * 32 + 1), f(c * 32 + 2));
#pragma unroll
                        for (int i = 3; i < 31; i += 2) a = max3(a, f(c * 32 + i), f(c * 32 + i + 1));
                        tops[c] = fmaxf(a, f(c * 32 + 31));
                    }
                    const float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
                    if (__any_sync(0xffffffffu, top > mx + by)) {
                        const float now = fmaxf(mx, top);
                        const float g = mx == now ? 1.f : ex2((mx - now) * p.scale_log2);   // (-inf before the first score: 0)
                        mx = now;
                        l *= g;
                        if (v >= 2) {   // (the products before this tile's scores are done)
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(tO + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * g);
                                tmem_st16(tO + c, o);
                            }
                            tmem_wait_st();
                        }
                    }
                    // The difference to the maximum is taken before the scaling: whatever the scores' size, it is as exact as they are.
                    const float from = mx == -INFINITY ? 0.f : -mx;
                    const float2 from2 = make_float2(from, from), sc = make_float2(p.scale_log2, p.scale_log2);
                    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t pk[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float2 x = __fmul2_rn(__fadd2_rn(make_float2(f(c * 32 + 2 * i), f(c * 32 + 2 * i + 1)), from2), sc);
                            const float2 e = make_float2(ex2(x.x), ex2(x.y));
                            sum = __fadd2_rn(sum, e);
                            pk[i] = pack(e.x, e.y);
                        }
                        tmem_st16(tS + c * 16, pk);
                        if (c == 1) {
                            tmem_wait_st();
                            tc_fence_before();
                            mbar_arrive(bar(&m->p_full[slot][0]));
                        }
                    }
                    l += sum.x + sum.y;
                    tmem_wait_st();
                } else {
                    tc_fence_before();
                    mbar_arrive(bar(&m->p_full[slot][0]));
                }
                tc_fence_before();
                mbar_arrive(bar(&m->p_full[slot][1]));
            }
            // The next unit's queries, when this one's last scores are done; then this one's results.
            const Walk x = k;
            wait(bar(&m->q_empty), x.seg & 1, abort_s);
            more = k.next(p, list, seqs, lane);
            if (more) load_queries(k);
            const bool slot_has[2] = {true, x.visits > 1};
            float2 other = make_float2(-INFINITY, 0.f);
            if (!x.wide) {
                ml_s[slot * 128 + row] = make_float2(live ? mx : -INFINITY, l);
                softmax_barrier();
                other = ml_s[(slot ^ 1) * 128 + row];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (!slot_has[i]) continue;
                // (a wide unit's slot needs its own alone, but both keep count of both)
                wait(bar(&m->o_full[i]), o_parity[i], abort_s);
                o_parity[i] ^= 1;
            }
            tc_fence_after();
            int flag = *(volatile int32_t *)&m->flags[x.seg & (kAhead - 1)];
            const bool poison = *(volatile int32_t *)&m->poison[x.seg & (kAhead - 1)] != 0;
            if (*abort_s || (int)blockIdx.x == p.give_up) flag |= kGaveUp;
            // weights of the slots' results; a narrow unit's slot writes half of the columns
            float w_own = 1.f, w_other = 0.f;
            if (!x.wide) {
                const float now = fmaxf(live ? mx : -INFINITY, other.x);
                w_own = mx == now ? 1.f : (mx == -INFINITY || !live) ? 0.f : ex2((mx - now) * p.scale_log2);
                w_other = other.x == -INFINITY ? 0.f : other.x == now ? 1.f : ex2((other.x - now) * p.scale_log2);
                if (mx == -INFINITY) w_own = 0.f;
                l = l * w_own + other.y * w_other;
                mx = now;
            }
            const int col0 = x.wide ? 0 : slot * (D / 2), col1 = x.wide ? D : col0 + D / 2;
            const uint32_t tOwn = tmem + kTmemO + (x.wide ? slot * D : 0) + lane_base, tOther = tmem + kTmemO + D + lane_base;
            // narrow: slot 0's result with its weight, then slot 1's
            const float w0 = x.wide ? 1.f : slot == 0 ? w_own : w_other, w1 = slot == 0 ? w_other : w_own;
            const size_t orow = ((size_t)x.u.b * p.T + node) * p.Hq + x.u.h * p.G + (grow - node * p.G);
            const int share = 2 * blockIdx.x + (x.u.t0 == 0 ? 1 : 0);
            const size_t srow = (size_t)share * 256 + (x.wide ? slot * 128 : 0) + row;
            const float inv = flag || l == 0.f ? 0.f : 1.f / l;   // (a row that sees nothing: zeros)
            if (warp_live) {
#pragma unroll 1
                for (int c = col0; c < col1; c += 16) {
                    uint32_t o[16], o1[16];
                    tmem_ld16(tOwn + c, o);
                    if (!x.wide && slot_has[1]) tmem_ld16(tOther + c, o1);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float y = __uint_as_float(o[i]) * w0;
                        if (!x.wide && slot_has[1]) y = fmaf(__uint_as_float(o1[i]), w1, y);
                        o[i] = __float_as_uint(y);
                    }
                    if (poison && has_tree && live) {   // infinities and NaN were left out of the product: the rows that see them get them
                        for (int n = 0; n < p.T; ++n) {
                            bool sees = false;
                            if (p.anc) sees = (p.anc[((size_t)x.u.b * p.T + node) * 2 + (n >> 6)] >> (n & 63)) & 1;
                            else for (int i = node; i != -1; i = p.parent[(size_t)x.u.b * p.T + i]) {
                                if (i == n) sees = true;
                                if (flag & kBadTree) break;
                            }
                            if (!sees) continue;
                            const __nv_bfloat16 *val = p.v_tree + (((size_t)x.u.b * p.T + n) * p.Hkv + x.u.h) * D + c;
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t bits = (uint32_t)*reinterpret_cast<const uint16_t *>(val + i) << 16;
                                if (nonfinite(bits)) {
#pragma unroll
                                    for (int e = 0; e < 16; ++e)
                                        if (e == i) o[e] = __float_as_uint(__uint_as_float(o[e]) + __uint_as_float(bits));
                                }
                            }
                        }
                    }
                    if (!live) continue;
                    if (x.whole) {
                        uint4 y[2];
                        uint32_t *w = reinterpret_cast<uint32_t *>(y);
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = flag ? 0u : pack(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
                        uint4 *dst = reinterpret_cast<uint4 *>(p.out + orow * D + c);
                        dst[0] = y[0];
                        dst[1] = y[1];
                    } else {
                        uint4 *dst = reinterpret_cast<uint4 *>(p.partial_o + srow * D + c);
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                }
                if (live && (x.wide || slot == 0)) {
                    if (!x.whole) p.partial_ml[srow] = make_float2(mx, l);
                    else if (p.lse) p.lse[orow] = flag ? 0.f : fmaf(mx, p.scale, log2f(l) * 0.6931471805599453f);
                }
            }
            tc_fence_before();
            softmax_barrier();   // both slots have read what the next unit's value products and results will overwrite
            if (tid == 0) {
                m->flags[x.seg & (kAhead - 1)] = 0;
                m->poison[x.seg & (kAhead - 1)] = 0;
                if (x.whole) {
                    note(p, x.u.b, flag, 0);
                } else {
                    p.flags[share] = flag;
                    const int c0 = list.worker_of(x.u.first_entry(kUnitCost)), c1 = list.worker_of(x.u.last_entry(kUnitCost));
                    m->task[share & 1] = ShareTask{x.u.b, x.u.h, x.u.rt, x.rows, c0, c1};
                }
            }
            trees += has_tree;
        }
        // Units that other blocks have shares of: at most one that goes on from the block before, one that goes on in the next.
        softmax_barrier();
        if (tid < 2 && m->task[tid].block0 >= 0) {
            __threadfence();
            if (atomicAdd(p.counters + m->task[tid].block0, 1) == m->task[tid].block1 - m->task[tid].block0) {
                __threadfence();
                m->last[tid] = 1;
            }
        }
        softmax_barrier();
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            if (!m->last[i]) continue;
            const ShareTask t = m->task[i];
            const int count = t.block1 - t.block0 + 1;
            auto slot_of = [&](int n) { return 2 * (t.block0 + n) + (n == 0 ? 1 : 0); };
            int flag = 0;
            for (int n = lane; n < count; n += 32) flag |= __ldcg(p.flags + slot_of(n));
            flag = __reduce_or_sync(0xffffffffu, flag);
            if (warp == 0) note(p, t.b, flag, lane);
            for (int r = warp; r < t.rows; r += 8) {
                const int g = t.rt * 256 + r, j = node_of(p, g);
                const Row y = merge_row<D>(
                    count, p.scale_log2, [&](int n) { return __ldcg(p.partial_ml + (size_t)slot_of(n) * 256 + r); },
                    [&](int n) { return __ldcg(reinterpret_cast<const float4 *>(p.partial_o + ((size_t)slot_of(n) * 256 + r) * D + lane * 4)); });
                put_row<D>(p, ((size_t)t.b * p.T + j) * p.Hq + t.h * p.G + (g - j * p.G), y, flag);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

}  // namespace

reader_status launch_q4_attn_sm100(Q4AttrSet *attr, const Q4AttnParams &params, int n_sm, cudaStream_t st) {
    Q4AttnParams p = params;
    bool &set = attr->sm100[p.D == 128];
    if (!set) {
        if (cudaFuncSetAttribute(p.D == 128 ? q4_attn_sm100_kernel<128> : q4_attn_sm100_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 p.D == 128 ? Cfg<128>::kSmem : Cfg<64>::kSmem) != cudaSuccess) {
            cudaGetLastError();
            return READER_ERR_CUDA;
        }
        set = true;
    }
    p.n_ctas = n_sm;
    launch_q4_attn_zero(p, n_sm, st);
    launch_pdl(p.D == 128 ? q4_attn_sm100_kernel<128> : q4_attn_sm100_kernel<64>, dim3((unsigned)n_sm), dim3(kThreads),
               (size_t)(p.D == 128 ? Cfg<128>::kSmem : Cfg<64>::kSmem), st, p);
    return READER_OK;
}

}  // namespace reader

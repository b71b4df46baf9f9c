// Tree-masked attention over a 4-bit cache for many query rows (reader_q4_verify_attn): draft trees, on the tcgen05 tensor cores.
//
// Bound: the tensor pipe and the exponentials, 2048 cycles each for 256 query rows and 128 keys; what 4 bits add is turning
// numbers into bf16 operands, 16384 of them for each, once for all rows that share them.  So a thread block (one per SM) has up to
// 256 rows of one KV head, two slots of 128, and eight warps of it do nothing but unpack: a tile of 128 keys (two pages) becomes
// the rows of K, and its values the rows of V^T (position pairs are neighbours in the pages, so a pair of numbers is a
// pair of bf16 along the value product's inner axis as it stands), in the 128-byte swizzle of the matrix instructions.
//
//   warps 0-3, 4-7   softmax of slot 0 and 1: a thread per row.  Scores come from tensor memory; the maximum in use is raised when a
//                    score exceeds it by 2^8 (O is rescaled in tensor memory then); probabilities replace the scores as bf16 and are the
//                    value product's A operand from there.  At a unit's end they fetch the next one's queries, so that its first
//                    products run beside the results being written.
//   warps 8-15       unpack pages (and copy the tree's own keys and values) into the tiles
//   warp 16          brings pages into a ring by bulk copies
//   warps 17, 18     issue the products of slot 0 and 1: S = Q K^T, O += P V.  In a wide piece they take turns with their score products,
//                    and slot 1 begins half a step late: left to themselves the slots fall into step, both at the exponentials and
//                    then both at the products
//   warp 19          finds the block's units and puts them into a small ring that the others read; zero rows for sequences whose
//                    length cannot be.  (With the search in every role the code did not fit the instruction caches any more, and
//                    warps stood waiting for instructions.)
// A unit of more than 128 rows is wide: each slot has its own rows and both work on every tile.  A narrow one has up to 128 rows;
// the slots take the tiles in turns and their two results are merged at its end.
//
// Tensor memory: S of either slot (128 columns each; P over its first 64), O of either slot.  The products of a slot are issued by one
// thread and run in order, so S[i + 1] may be written over P[i] as soon as the value product that reads it has been issued.
//
// Work: a flat list of tiles cut into equal ranges, one per thread block (q4_attn_common.cuh); shares of units in several ranges are merged by
// a launch behind.  Bytes that are not committed never reach a product: their scores become -inf, and their values 0 or
// not multiplied at all (16-key slices behind the end).  Every wait is bounded: a block that gives up reports all its units.
#include <algorithm>
#include <type_traits>

#include "prompt_ptx.cuh"
#include "q4_attn_common.cuh"

namespace reader {
namespace {

using namespace q4;

constexpr int kThreads = 640;
constexpr int kSoftmaxThreads = 256;
constexpr int kUnpackWarp = 8, kLoadWarp = 16, kMmaWarp = 17, kListWarp = 19;
constexpr int kUnpackThreads = 256, kUnpackWarps = 8;
constexpr int kReaders = 19;       // warps that read the ring of units: all but kListWarp
// Registers of a thread: softmax, unpacking, the rest: 256 x 112 + 256 x 72 + 128 x 96 = 59392 of the 640 x 96 that the block is launched with.
constexpr int kRegsSoftmax = 112, kRegsUnpack = 72;
constexpr int kLateStart = 6;      // tiles of a wide piece from which slot 1 begins half a step behind slot 0
constexpr int kTileKeys = 128;     // keys of a tile: two pages
constexpr int kUnitCost = 6;       // entries that stand for a unit's start and end
constexpr int kMinEntries = 8;     // of a range
constexpr int kRawSlots = 3;       // of the ring: keys or values of a tile's pages each
constexpr int kAhead = 8;          // units in the ring
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
    static constexpr int kSmem = kOffBars + 1024;
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

// A unit as the roles see it: its tiles t0 .. t0 + tiles - 1 are this block's.
struct Piece {
    int b, h, rt, L, npages, ntiles, t0, tiles;   // tiles = 0: no more units
    int wide, rows, last;                         // rows of the unit; the block that has its last tile
    __device__ __forceinline__ bool whole() const { return tiles == ntiles; }
    // committed tiles come first, the tree's is the last
    __device__ __forceinline__ bool is_tree(int tile) const { return t0 + tile == ntiles - 1; }
    __device__ __forceinline__ int valid(int T, int tile) const { return is_tree(tile) ? T : min(kTileKeys, L - (t0 + tile) * kTileKeys); }
    // tiles of a slot: every one, or (narrow) every other
    __device__ __forceinline__ int first(int slot) const { return wide ? 0 : slot; }
    __device__ __forceinline__ int step() const { return wide ? 1 : 2; }
};
struct Bars {
    uint64_t raw_full[kRawSlots], raw_empty[kRawSlots], k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t q_full, q_empty, s_full[2], p_full[2][2], o_full[2], turn[2], piece_full[kAhead], piece_empty[kAhead];
    uint32_t tmem_base;
    int32_t abort;
    int32_t raw_bad[kRawSlots];   // a page outside the pool among the slot's
    int32_t flags[kAhead];        // what is wrong with unit i mod kAhead
    int32_t poison[kAhead];       // its tree has infinities or NaN among the values
    int32_t warp_sum[kThreads / 32];
    ShareTask task;               // the unit that this block begins and others go on with
    Piece piece[kAhead];
};
static_assert(sizeof(Bars) <= 1024, "barrier block");

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

// Among the softmax threads and kListWarp.
template <int kId>
__device__ __forceinline__ void end_barrier() { asm volatile("bar.sync %0, %1;" ::"n"(kId), "n"(kSoftmaxThreads + 32) : "memory"); }
// Unit number `seg` from the ring, for a whole warp; false when there is none, or when the block has given up.
__device__ __forceinline__ bool next_piece(Bars *m, Piece &x, int seg, int lane, volatile int32_t *abort_s) {
    const int i = seg % kAhead;
    if (!wait(smem_u32(&m->piece_full[i]), (seg / kAhead) & 1, abort_s)) return false;
    x = m->piece[i];
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&m->piece_empty[i]));
    return x.tiles > 0;
}

// ---- unpacking (`t`: among the 128 threads of a page)
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
    constexpr int kWordsHere = 8 / kSplit;
    uint32_t word[kWordsHere];
#pragma unroll
    for (int j = 0; j < kWordsHere; ++j) word[j] = lds32(src + j * 8 * (D / 2));
    const uint32_t odd = kPer == 2 ? (u & 1) * 0x0101u : 0u;
    auto go = [&](auto whole) {
#pragma unroll
        for (int j = 0; j < kWordsHere; ++j) {
            constexpr bool kWhole = decltype(whole)::value;
            const uint32_t sel = 0x4040u | (j * kPer & 3) * 0x0101u;
            const Scale2 s = scale2<kWhole>(__byte_perm(codes[j * kPer >> 2], 0, sel + odd));
            sts128(dst + j * 8 * 128, pair<0>(word[j], s, sixteen), pair<1>(word[j], s, sixteen), pair<2>(word[j], s, sixteen), pair<3>(word[j], s, sixteen));
        }
    };
    if (nan_bits(codes[0]) | nan_bits(codes[1]) | nan_bits(codes[2]) | nan_bits(codes[3])) go(std::false_type());
    else go(std::true_type());
}
// A page of values into a page of V^T, `valid` of its positions committed (the others become 0).  Thread (q, z, f): the positions 8 q .. + 7 of half f
// of the elements z D/8 .. + D/8 - 1.
template <int D>
__device__ __forceinline__ void unpack_values(uint32_t raw, uint32_t page, int valid, int t, uint32_t sixteen) {
    constexpr int kWords = D / 64;
    const int q = t & 7, z = (t >> 3) & 7, f = t >> 6;
    if (8 * q >= ((valid + 15) & ~15)) return;   // (behind the last slice that is multiplied)
    // The four position pairs 4 q + e, each lane's in an order that begins with e = q mod 4 (in one order for all, eight lanes would meet in
    // the same banks): k-th load e = (k + q) mod 4.
    uint32_t w[4][kWords], codes[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int e = (k + q) & 3, pr = 4 * q + e;
        const uint32_t at = raw + pr * D + v_chunk<D>(pr, z) * (D / 8) + f * (D / 16);
        if constexpr (D == 128) { const uint2 x = lds64(at); w[k][0] = x.x; w[k][1] = x.y; }
        else w[k][0] = lds32(at);
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
    const uint32_t both01 = codes[0] | codes[1] << 16, both23 = codes[2] | codes[3] << 16;
    if (8 * q + 8 <= valid && !(nan_bits(both01) | nan_bits(both23))) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] = scale2<true>(__byte_perm(codes[e], 0, 0x4140));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[e] = scale2<false>(__byte_perm(codes[e], 0, 0x4140));
            const int key = 8 * q + 2 * e;
            if (key >= valid) { s[e].s &= 0xffff0000u; s[e].m24 &= 0xffff0000u; }
            if (key + 1 >= valid) { s[e].s &= 0xffffu; s[e].m24 &= 0xffffu; }
        }
    }
#pragma unroll
    for (int y = 0; y < kWords; ++y) {
        // row d = z D/8 + f D/16 + 4 y + i
        const uint32_t rows = page + (z * (D / 8) + f * (D / 16)) * 128;
        const int turn = D == 128 ? 0 : 4 * f;   // (of the row's number, what its place in the swizzle goes by)
        auto row = [&](int i) { return rows + (4 * y + i) * 128 + ((q ^ ((turn + 4 * y + i) & 7)) << 4); };
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
    for (int i = t; i < p.T * kChunks; i += kUnpackThreads) {
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
    for (int i = t; i < groups * kChunks; i += kUnpackThreads) {
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
            mbar_init(bar(&m->raw_empty[i]), kUnpackWarps);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&m->k_full[i]), kUnpackWarps);
            mbar_init(bar(&m->k_empty[i]), 2);
            mbar_init(bar(&m->v_full[i]), kUnpackWarps);
            mbar_init(bar(&m->turn[i]), 1);
            mbar_init(bar(&m->v_empty[i]), 2);
            mbar_init(bar(&m->s_full[i]), 1);
            mbar_init(bar(&m->p_full[i][0]), 128);
            mbar_init(bar(&m->p_full[i][1]), 128);
            mbar_init(bar(&m->o_full[i]), 1);
        }
        m->task.block0 = -1;
        mbar_init(bar(&m->q_full), kSoftmaxThreads);
        mbar_init(bar(&m->q_empty), 2);
        for (int i = 0; i < kAhead; ++i) {
            mbar_init(bar(&m->piece_full[i]), 1);
            mbar_init(bar(&m->piece_empty[i]), kReaders);
            m->flags[i] = m->poison[i] = 0;
        }
        m->abort = (base & 1023u) ? 1 : 0;   // (the swizzled tiles want 1024-byte alignment; never seen otherwise, but checked)
        fence_mbar_init();
        fence_proxy_async();
        mbar_arrive(bar(&m->turn[0]));   // slot 0 has the first turn
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

    if (warp >= kLoadWarp) {
        if (warp == kListWarp) {
            // ------------------------------------------------------------------ units
            int w = 0, w_end = 0;
            if ((int)blockIdx.x < list.n_workers && list.W > 0) {
                w = list.begin(blockIdx.x);
                w_end = list.begin(blockIdx.x + 1);
            }
            for (int seg = 0;; ++seg) {
                Piece x{};
                while (w < w_end) {
                    const Unit u = unit_at(p, list, seqs, w, w_end, lane);
                    w += u.entries;
                    if (!u.any) continue;
                    x = Piece{u.b, u.h, u.rt, u.L, u.npages, u.ntiles, u.t0, u.t1 - u.t0, u.weight == 2, min(256, p.T * p.G - u.rt * 256), 0};
                    if (!x.whole()) x.last = list.worker_of(u.last_entry(kUnitCost));
                    break;
                }
                const int i = seg % kAhead;
                if (!wait(bar(&m->piece_empty[i]), ((seg / kAhead) & 1) ^ 1, abort_s)) break;
                if (lane == 0) {
                    m->piece[i] = x;
                    mbar_arrive(bar(&m->piece_full[i]));
                }
                __syncwarp();
                if (x.tiles == 0) break;
            }
            reject_lengths<D>(p, blockIdx.x, gridDim.x, lane);
            end_barrier<3>();
            if (gone(abort_s) && (int)blockIdx.x < list.n_workers && list.W > 0) {
                // The block has given up: whatever became of its units, whole ones are zeroed and reported, shares are reported to those who merge.
                w = list.begin(blockIdx.x);
                while (w < w_end) {
                    const Unit u = unit_at(p, list, seqs, w, w_end, lane);
                    w += u.entries;
                    if (!u.any) continue;
                    const int rows = min(256, p.T * p.G - u.rt * 256);
                    if (u.t0 == 0 && u.t1 == u.ntiles) {
                        note(p, u.b, kGaveUp, lane);
                        for (int r = 0; r < rows; ++r) {
                            const int g = u.rt * 256 + r, j = node_of(p, g);
                            put_row<D>(p, ((size_t)u.b * p.T + j) * p.Hq + u.h * p.G + (g - j * p.G), Row{0.f, 1.f, make_float4(0.f, 0.f, 0.f, 0.f)}, kGaveUp);
                        }
                    } else if (lane == 0) {
                        const int i = u.t0 == 0 ? 1 : 0;
                        p.flags[2 * blockIdx.x + i] = kGaveUp;
                        if (i) m->task = ShareTask{u.b, u.h, u.rt, rows, (int)blockIdx.x, list.worker_of(u.last_entry(kUnitCost))};
                    }
                }
            }
            end_barrier<4>();
        } else
        if (warp == kLoadWarp) {
            // ------------------------------------------------------------------ pages
            const uint64_t policy = l2_policy_evict_first();
            const bool once = list.n_wide + list.narrow == 1;   // no other unit reads these pages
            int n = 0;   // slots of the ring so far
            Piece x;
            for (int seg = 0; next_piece(m, x, seg, lane, abort_s); ++seg) {
                const int pages_end = min(x.npages, 2 * (x.t0 + x.tiles));
                int ids = 0, at = -32;
                for (int t = 0; t < x.tiles && !gone(abort_s); ++t) {
                    if (x.is_tree(t)) break;
                    const int page0 = 2 * (x.t0 + t);
                    if (page0 - at >= 32) {
                        at = page0;
                        ids = page0 + lane < pages_end ? p.page_table[(size_t)x.b * p.max_pages + page0 + lane] : 0;
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
                            if (ok0) bulk_load(dst, pool + ((size_t)id0 * p.Hkv + x.h) * C::kPageBytes, C::kPageBytes, full, policy, streamed);
                            if (count == 2 && ok1) bulk_load(dst + C::kPageBytes, pool + ((size_t)id1 * p.Hkv + x.h) * C::kPageBytes, C::kPageBytes, full, policy, streamed);
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
        } else {
            // ------------------------------------------------------------------ products of a slot
            const int slot = warp - kMmaWarp;
            constexpr uint32_t kIdescQK = idesc_bf16_f32(128, kTileKeys, false, false), kIdescPV = idesc_bf16_f32(128, D, false, false);
            const uint64_t descQ = smem_desc_sw128(base + C::kOffQ, 16, 1024), descK = smem_desc_sw128(base + C::kOffK, 16, 1024);
            const uint64_t descV = smem_desc_sw128(base + C::kOffV, 16, 1024);
            const uint32_t tS = tmem + kTmemS + slot * 128, tO = tmem + kTmemO + slot * D;
            // Both issuers see every tile of keys and of values in order, so that neither can fall a whole turn behind (a parity wait tells
            // a phase only from the one before it); tiles of the other slot are passed on at once.
            int nk = 0, nv = 0, done = 0;   // tiles of keys, of values seen; of the units before
            uint32_t p_parity = 0, turn_parity = 0;
            auto pass_keys = [&](int to) {
                for (; nk < to; ++nk) {
                    wait(bar(&m->k_full[nk & 1]), (nk >> 1) & 1, abort_s);
                    if (lane == 0) mbar_arrive(bar(&m->k_empty[nk & 1]));
                    __syncwarp();
                }
            };
            auto pass_values = [&](int to) {
                for (; nv < to; ++nv) {
                    wait(bar(&m->v_full[nv & 1]), (nv >> 1) & 1, abort_s);
                    if (lane == 0) mbar_arrive(bar(&m->v_empty[nv & 1]));
                    __syncwarp();
                }
            };
            Piece x;
            for (int seg = 0; next_piece(m, x, seg, lane, abort_s); ++seg) {
                wait(bar(&m->q_full), seg & 1, abort_s);
                const int step = x.step();
                const uint64_t qd = descQ + (uint64_t)((x.wide ? slot * C::kQBytes : 0) >> 4);
                const bool late = x.wide && slot == 0 && x.tiles >= kLateStart;
                auto pass_turn = [&]() {
                    if (x.wide && lane == 0) mbar_arrive(bar(&m->turn[slot ^ 1]));
                    __syncwarp();
                };
                auto score = [&](int t) {
                    pass_keys(done + t);
                    const int buf = nk & 1;
                    wait(bar(&m->k_full[buf]), (nk >> 1) & 1, abort_s);
                    ++nk;
                    if (x.wide) {
                        wait(bar(&m->turn[slot]), turn_parity, abort_s);
                        turn_parity ^= 1;
                    }
                    tc_fence_after();
                    const bool go = !gone(abort_s);
                    if (go && elect_one()) {
                        const uint64_t kd = descK + (uint64_t)((buf * C::kKBytes) >> 4);
#pragma unroll
                        for (int hf = 0; hf < C::kHalves; ++hf)
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                mma_bf16_ss(tS, qd + (uint64_t)((hf * C::kBlock + kk * 32) >> 4), kd + (uint64_t)((hf * C::kBlock + kk * 32) >> 4), kIdescQK, (hf | kk) != 0);
                        mma_commit(bar(&m->s_full[slot]));
                        mma_commit(bar(&m->k_empty[buf]));
                        if (t + step >= x.tiles) mma_commit(bar(&m->q_empty));
                    }
                    __syncwarp();
                    if (!(late && t == 0)) pass_turn();
                };
                const int t0 = x.first(slot);
                if (t0 < x.tiles) {
#pragma unroll 1
                    for (int t = t0 - step; t < x.tiles; t += step) {
                        if (t >= t0) {
                            pass_values(done + t);
                            const int buf = nv & 1, slices = (x.valid(p.T, t) + 15) >> 4;
                            wait(bar(&m->v_full[buf]), (nv >> 1) & 1, abort_s);
                            ++nv;
#pragma unroll 1
                            for (int half = 0; half < 2; ++half) {
                                wait(bar(&m->p_full[slot][half]), p_parity, abort_s);
                                if (late && t == 0 && half == 0) pass_turn();
                                tc_fence_after();
                                const bool go = !gone(abort_s);
                                if (go && elect_one()) {
                                    const uint64_t vd = descV + (uint64_t)((buf * C::kVBytes + half * C::kVPage) >> 4);
#pragma unroll
                                    for (int kk = 0; kk < 4; ++kk)
                                        if (half * 4 + kk < slices)
                                            mma_bf16_ts(tO, tS + (half * 4 + kk) * 8, vd + (uint64_t)((kk * 32) >> 4), kIdescPV, t != t0 || half + kk != 0);
                                    if (half == 1) {
                                        mma_commit(bar(&m->v_empty[buf]));
                                        if (t + step >= x.tiles) mma_commit(bar(&m->o_full[slot]));
                                    }
                                }
                                __syncwarp();
                            }
                            p_parity ^= 1;
                        }
                        if (t + step < x.tiles) score(t + step);
                    }
                } else {   // (a narrow piece of one tile: slot 1 has none)
                    if (lane == 0) mbar_arrive(bar(&m->q_empty));
                    __syncwarp();
                }
                done += x.tiles;
                pass_keys(done);
                pass_values(done);
            }
            if (gone(abort_s)) __nanosleep(1000000);   // products that are still under way end before their operands go away
        }
    } else if (warp >= kUnpackWarp) {
        // ------------------------------------------------------------------ unpacking
        regs_dec<kRegsUnpack>();
        const int t = tid - kUnpackWarp * 32;
        volatile uint32_t *word = reinterpret_cast<volatile uint32_t *>(smem + C::kOffMl);   // (an opaque constant: see pair())
        if (t == 0) *word = 0x41804180u;
        asm volatile("bar.sync 2, 256;" ::: "memory");
        const uint32_t sixteen = *word;
        asm volatile("bar.sync 2, 256;" ::: "memory");
        int n = 0, raw = 0, trees = 0;   // tiles, slots of the ring, trees so far
        Piece x;
        for (int seg = 0; next_piece(m, x, seg, lane, abort_s); ++seg) {
            for (int i = 0; i < x.tiles && !gone(abort_s); ++i, ++n) {
                const int buf = n & 1;
                const uint32_t kt = base + C::kOffK + buf * C::kKBytes, vt = base + C::kOffV + buf * C::kVBytes;
                const bool tree = x.is_tree(i);
                const int valid = x.valid(p.T, i);
                // keys
                if (!wait(bar(&m->k_empty[buf]), ((n >> 1) & 1) ^ 1, abort_s)) break;
                if (tree) {
                    unsigned char *parents = smem + C::kOffParents + (trees & (kAhead / 2 - 1)) * kMaxNodes;
                    if (t < p.T) {
                        const int a = p.parent[(size_t)x.b * p.T + t];
                        parents[t] = (unsigned char)a;
                        if (!(t == 0 ? a == -1 : a >= 0 && a < t)) atomicOr(&m->flags[seg & (kAhead - 1)], kBadTree);
                    }
                    copy_tree_keys<D>(p, x.b, x.h, kt, t);
                    ++trees;
                } else {
                    const int s = raw % kRawSlots;
                    if (!wait(bar(&m->raw_full[s]), (raw / kRawSlots) & 1, abort_s)) break;
                    const uint32_t src = base + C::kOffRaw + s * C::kRawBytes;
                    if (m->raw_bad[s] && t == 0) atomicOr(&m->flags[seg & (kAhead - 1)], kBadPage);
                    const int page = t >> 7;   // a page to 128 threads
                    if (page * kPage < valid) unpack_keys<D>(src + page * C::kPageBytes, kt, page * kPage, t & 127, sixteen);
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
                    if (copy_tree_values<D>(p, x.b, x.h, vt, t)) atomicOr(&m->poison[seg & (kAhead - 1)], 1);
                } else {
                    const int s = raw % kRawSlots;
                    if (!wait(bar(&m->raw_full[s]), (raw / kRawSlots) & 1, abort_s)) break;
                    const uint32_t src = base + C::kOffRaw + s * C::kRawBytes;
                    const int page = t >> 7;
                    if (page * kPage < valid) unpack_values<D>(src + page * C::kPageBytes, vt + page * C::kVPage, min(valid - page * kPage, kPage), t & 127, sixteen);
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
        auto load_queries = [&](const Piece &x) {
            const int r = x.rt * 256 + (x.wide ? slot * 128 : 0) + row;
            const bool live = r < p.T * p.G;
            const int j = live ? node_of(p, r) : 0, hq = x.h * p.G + (live ? r - j * p.G : 0);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (((size_t)x.b * p.T + j) * p.Hq + hq) * D);
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
        // Whether there is another unit is decided together: a block that gives up may do so between two warps' looks at the ring, and the
        // barriers among the softmax threads want all of them.
        auto next_for_all = [&](Piece &y, int seg) {
            const bool got = next_piece(m, y, seg, lane, abort_s);
            int all;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 256, p;\n\tselp.b32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"((int)got) : "memory");
            return all != 0;
        };
        Piece k;
        int seg = 0;
        bool more = next_for_all(k, 0);
        if (more) load_queries(k);
        while (more) {
            const int grow = k.rt * 256 + (k.wide ? slot * 128 : 0) + row;   // among the head's rows
            const bool live = grow < p.T * p.G;
            const bool warp_live = __any_sync(0xffffffffu, live);
            const int node = live ? node_of(p, grow) : 0;
            // a row without a query never asks for a higher maximum
            float mx = live ? -INFINITY : INFINITY, l = 0.f;
            const bool has_tree = k.is_tree(k.tiles - 1);
            const int t_first = k.first(slot);
#pragma unroll 1
            for (int t = t_first; t < k.tiles; t += k.step()) {
                wait(bar(&m->s_full[slot]), s_parity, abort_s);
                s_parity ^= 1;
                tc_fence_after();
                if (warp_live) {
                    const int valid = k.valid(p.T, t);
                    const bool masked = valid < kTileKeys || k.is_tree(t);
                    uint64_t sees[2] = {~0ull, ~0ull};   // the keys this row sees
                    if (masked) {
                        if (k.is_tree(t)) {
                            sees[0] = sees[1] = 0;
                            if (live && p.anc) {
                                sees[0] = p.anc[((size_t)k.b * p.T + node) * 2];
                                sees[1] = p.anc[((size_t)k.b * p.T + node) * 2 + 1];
                            } else if (live && !(*(volatile int32_t *)&m->flags[seg % kAhead] & kBadTree)) {
                                const unsigned char *parents = smem + C::kOffParents + (trees & (kAhead / 2 - 1)) * kMaxNodes;
                                for (int i = node; i != 255; i = parents[i]) {   // (strictly falling on a valid tree)
                                    if (i < 64) sees[0] |= 1ull << i;
                                    else sees[1] |= 1ull << (i - 64);
                                }
                            }
                        }
                        if (valid < 64) sees[0] &= (1ull << valid) - 1;
                        if (valid < 128) sees[1] &= valid <= 64 ? 0 : (1ull << (valid - 64)) - 1;
                    }
                    // Half a tile's scores at a time, twice: for the maximum, then for the probabilities.  (All 128 in registers leave none
                    // for the warps that unpack; tensor memory is read in a fraction of the time that the exponentials take.)
                    uint32_t x[2][32];
                    auto f = [&](int i) { return __uint_as_float(x[i >> 5][i & 31]); };
                    auto fetch = [&](int half) {
                        tmem_ld32(tS + half * 64, x[0]);
                        tmem_ld32(tS + half * 64 + 32, x[1]);
                        tmem_wait_ld();
                        if (masked) {
                            const uint64_t bits = sees[half];
#pragma unroll
                            for (int i = 0; i < 64; ++i)
                                if (!((bits >> i) & 1)) x[i >> 5][i & 31] = kNegInf;
                        }
                    };
                    float top = -INFINITY;
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {
                        fetch(half);
                        float a = max3(f(0), f(1), f(2)), b = max3(f(3), f(4), f(5));
#pragma unroll
                        for (int i = 6; i < 62; i += 4) {
                            a = max3(a, f(i), f(i + 1));
                            b = max3(b, f(i + 2), f(i + 3));
                        }
                        top = fmaxf(top, fmaxf(max3(a, f(62), f(63)), b));
                    }
                    if (__any_sync(0xffffffffu, top > mx + by)) {
                        const float now = fmaxf(mx, top);
                        const float g = mx == now ? 1.f : ex2((mx - now) * p.scale_log2);   // (-inf before the first score: 0)
                        mx = now;
                        l *= g;
                        if (t != t_first) {   // (the products before this tile's scores are done)
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
#pragma unroll 1
                    for (int half = 0; half < 2; ++half) {   // (P of a half is written over scores that have been read)
                        fetch(half);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float2 y = __fmul2_rn(__fadd2_rn(make_float2(f(c * 32 + 2 * i), f(c * 32 + 2 * i + 1)), from2), sc);
                                const float2 e = make_float2(ex2(y.x), ex2(y.y));
                                sum = __fadd2_rn(sum, e);
                                pk[i] = pack(e.x, e.y);
                            }
                            tmem_st16(tS + half * 32 + c * 16, pk);
                        }
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive(bar(&m->p_full[slot][half]));
                    }
                    l += sum.x + sum.y;
                } else {
                    tc_fence_before();
                    mbar_arrive(bar(&m->p_full[slot][0]));
                    mbar_arrive(bar(&m->p_full[slot][1]));
                }
            }
            // The next unit's queries, when this one's last scores are done; then this one's results.
            const Piece x = k;
            const int seg_x = seg++;
            wait(bar(&m->q_empty), seg_x & 1, abort_s);
            more = next_for_all(k, seg);
            if (more) load_queries(k);
            const bool slot_has[2] = {true, x.wide || x.tiles > 1};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (!slot_has[i]) continue;
                // (a wide unit's slot needs its own alone, but both keep count of both)
                wait(bar(&m->o_full[i]), o_parity[i], abort_s);
                o_parity[i] ^= 1;
            }
            tc_fence_after();
            int flag = *(volatile int32_t *)&m->flags[seg_x % kAhead];
            if (*abort_s || (int)blockIdx.x == p.give_up) flag |= kGaveUp;
            if (has_tree && *(volatile int32_t *)&m->poison[seg_x % kAhead] && (x.wide || slot == ((x.tiles - 1) & 1)) && warp_live) {
                // infinities and NaN were left out of the product: the rows that see them get them
#pragma unroll 1
                for (int n = 0; n < p.T && !(flag & kBadTree); ++n) {
                    bool sees = false;
                    if (live && p.anc) sees = (p.anc[((size_t)x.b * p.T + node) * 2 + (n >> 6)] >> (n & 63)) & 1;
                    if (live && !p.anc)
                        for (int i = node; i >= n; i = p.parent[(size_t)x.b * p.T + i]) sees |= i == n;
                    const uint32_t *val = reinterpret_cast<const uint32_t *>(p.v_tree + (((size_t)x.b * p.T + n) * p.Hkv + x.h) * D);
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        uint32_t o[16];
                        tmem_ld16(tO + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint32_t w = val[c / 2 + i];
                            if (sees && nonfinite(w << 16)) o[2 * i] = __float_as_uint(__uint_as_float(o[2 * i]) + bf16lo(w));
                            if (sees && nonfinite(w)) o[2 * i + 1] = __float_as_uint(__uint_as_float(o[2 * i + 1]) + bf16hi(w));
                        }
                        tmem_st16(tO + c, o);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
            }
            float2 other = make_float2(-INFINITY, 0.f);
            if (!x.wide) {
                ml_s[slot * 128 + row] = make_float2(live ? mx : -INFINITY, l);
                softmax_barrier();
                tc_fence_after();
                other = ml_s[(slot ^ 1) * 128 + row];
            }
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
            const size_t orow = ((size_t)x.b * p.T + node) * p.Hq + x.h * p.G + (grow - node * p.G);
            const int share = 2 * blockIdx.x + (x.t0 == 0 ? 1 : 0);
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
                    if (!live) continue;
                    if (x.whole()) {
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
                    if (!x.whole()) p.partial_ml[srow] = make_float2(mx, l);
                    else if (p.lse) p.lse[orow] = flag ? 0.f : fmaf(mx, p.scale, log2f(l) * 0.6931471805599453f);
                }
            }
            tc_fence_before();
            softmax_barrier();   // both slots have read what the next unit's value products and results will overwrite
            if (tid == 0) {
                m->flags[seg_x % kAhead] = 0;
                m->poison[seg_x % kAhead] = 0;
                if (x.whole()) {
                    note(p, x.b, flag, 0);
                } else {
                    p.flags[share] = flag;
                    if (share & 1) m->task = ShareTask{x.b, x.h, x.rt, x.rows, (int)blockIdx.x, x.last};
                }
            }
            trees += has_tree;
        }
        end_barrier<3>();
        end_barrier<4>();
        if (tid == 0) p.tasks[blockIdx.x] = m->task;
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
}

// Units that several blocks have shares of: eight rows of the one that block blockIdx.x of the attention begins, a warp to a row.  (A launch of its
// own: the block that came last did this at first, and took 25 us for the shares of 128 rows and 60 us for those of 256, the others waiting.)
template <int D>
__global__ void __launch_bounds__(256) q4_attn_merge_kernel(const __grid_constant__ Q4AttnParams p) {
    const int lane = threadIdx.x & 31, r = blockIdx.y * 8 + (threadIdx.x >> 5);
    pdl_wait();
    pdl_launch_dependents();
    const ShareTask t = p.tasks[blockIdx.x];
    if (t.block0 < 0 || r >= t.rows) return;
    const int count = t.block1 - t.block0 + 1;
    auto slot_of = [&](int n) { return 2 * (t.block0 + n) + (n == 0 ? 1 : 0); };
    int flag = 0;
    for (int n = lane; n < count; n += 32) flag |= p.flags[slot_of(n)];
    flag = __reduce_or_sync(0xffffffffu, flag);
    if (r == 0) note(p, t.b, flag, lane);
    const int g = t.rt * 256 + r, j = node_of(p, g);
    const Row y = merge_row<D>(
        count, p.scale_log2, [&](int n) { return p.partial_ml[(size_t)slot_of(n) * 256 + r]; },
        [&](int n) { return *reinterpret_cast<const float4 *>(p.partial_o + ((size_t)slot_of(n) * 256 + r) * D + lane * 4); });
    put_row<D>(p, ((size_t)t.b * p.T + j) * p.Hq + t.h * p.G + (g - j * p.G), y, flag);
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
    launch_pdl(p.D == 128 ? q4_attn_merge_kernel<128> : q4_attn_merge_kernel<64>, dim3((unsigned)n_sm, (unsigned)((std::min(256, p.T * p.G) + 7) / 8)), dim3(256), 0,
               st, p);
    return READER_OK;
}

}  // namespace reader

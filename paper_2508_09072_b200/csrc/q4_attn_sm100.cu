// Tree-masked attention over a 4-bit cache for many query rows (reader_q4_verify_attn): draft trees, on the tcgen05 tensor cores.
//
// Bound: the tensor pipe and the exponentials, 2048 cycles each for 256 query rows and 128 keys; what 4 bits add is turning
// numbers into bf16 operands, 16384 of them for each, once for all rows that share them.  Measured (32 query heads, 8 KV heads, head_dim 128): four trees of 128
// nodes on 32768 positions 314 us, 0.88 PF/s; 32 trees of 32 nodes on 1024-4096 83 us.  Either way a step of 128 rows and 128 keys is 1.4 to 1.7 us,
// the softmax warps' 0.3 for the maximum and 0.85 to 1.05 for 16384 exponentials (0.54 if nothing else ran) and hardly a wait.  So a thread block (one per SM) has up to
// 256 rows of one KV head, two slots of 128, and eight warps of it do nothing but unpack: a tile of 128 keys (two pages) becomes
// the rows of K, and its values the rows of V^T (position pairs are neighbours in the pages, so a pair of numbers is a
// pair of bf16 along the value product's inner axis as it stands), in the 128-byte swizzle of the matrix instructions.
//
//   warps 0-7        softmax, all of them a step's 128 rows, two threads to a row, each with half of its keys: while they are at one slot's
//                    scores, the other's products run.  Scores come from tensor memory once; the maximum in use is raised when a score
//                    exceeds it by 2^8 (O is rescaled in tensor memory then), the one thing that a row's threads must agree on;
//                    probabilities replace the scores as bf16 and are the value product's A operand from there.  (A thread to a row and four
//                    warps to a slot: the tile's steps took 2.95 us, each slot's products waiting for its own exponentials and these for them.)
//   warps 8-11, 12-15  unpack pages (and copy the tree's own keys and values) into the tiles, every other tile each
//   warp 16          brings pages into a ring by bulk copies
//   warp 17          issues the products: S = Q K^T, O += P V
//   warp 18          brings queries
//   warp 19          finds the block's units and puts them into a small ring that the others read; zero rows for sequences whose
//                    length cannot be
//
// A step is 128 rows and a tile: of a unit of more than 128 rows (wide) the two slots of every tile, else (narrow) every tile, in the slots in turn.
// Products are issued by one thread and run in order, so S[i + 2] may be written over P[i] as soon as the value product that reads it
// has been issued.
//
// Work: a flat list of tiles cut into equal ranges, one per thread block (q4_attn_common.cuh); shares of units in several ranges are merged by
// a launch behind.  Bytes that are not committed never reach a product: their scores become -inf, and their values 0 or
// not multiplied at all (16-key slices behind the end).  Every wait is bounded: a block that gives up reports all its units.
#include <algorithm>
#include <type_traits>

#include "ancestors.cuh"
#include "prompt_ptx.cuh"
#include "q4_attn_common.cuh"

namespace reader {
namespace {

using namespace q4;

constexpr int kThreads = 640;
constexpr int kSoftmaxThreads = 256;
constexpr int kUnpackWarp = 8, kLoadWarp = 16, kMmaWarp = 17, kQueryWarp = 18, kListWarp = 19;
constexpr int kUnpackThreads = 128, kUnpackWarps = 4;   // of a tile
constexpr int kReaders = 19;       // warps that read the ring of units: all but kListWarp
// Registers of a thread: softmax, unpacking, the rest: 256 x 112 + 256 x 96 + 128 x 64 = the 640 x 96 that the block is launched with.  (24 bytes are spilled, 28 read
// back; at head_dim 64 20 and 24.)
constexpr int kRegsSoftmax = 112, kRegsUnpack = 96, kRegsRest = 64;
static_assert(2 * kRegsSoftmax + 2 * kRegsUnpack + kRegsRest <= 5 * 96 && kRegsSoftmax >= 96 && kRegsUnpack <= 96 && kRegsRest <= 96, "what a block is launched with");
constexpr int kTileKeys = 128;     // keys of a tile: two pages
constexpr int kUnitCost = 4;       // entries that stand for a unit's start and end (32 x 32 nodes, 4 x 128 on 32768: 82.8, 314 us; 2: 82.7, 316; 6: 84.8, 314)
constexpr int kMinEntries = kUnitCost + 2;   // of a range: so every one of them holds a tile
// Slots of the ring, keys or values of a tile's pages each: three, and three more in a call without wide units, in the half of the queries' place that it does
// not need (with three the narrow units' tiles come too late: 32 x 32 nodes 84.7 us, with six 82.9).
constexpr int kRawSlots = 3;
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
    static constexpr int kOffSwap = kOffParents + kAhead / 2 * kMaxNodes;   // what the two threads of a row tell each other: largest scores, sums
    static constexpr int kOffTable = kOffSwap + 2 * 256 * 4;
    static constexpr int kOffBars = kOffTable + kPrefix * 8;
    static constexpr int kSmem = kOffBars + 1024;
    static_assert(kSmem <= 227 * 1024 && kRawSlots * kRawBytes <= kQBytes, "shared memory");
    static __device__ __forceinline__ uint32_t raw_at(int s) { return s * kRawBytes + (s < kRawSlots ? kOffRaw : kOffQ + kQBytes - kRawSlots * kRawBytes); }
};

// A unit as the roles see it: its tiles t0 .. t0 + tiles - 1 are this block's.
struct Piece {
    int b, h, rt, L, npages, ntiles, t0, tiles;   // tiles = 0: no more units
    int wide, rows, last;                         // rows of the unit; the block that has its last tile
    __device__ __forceinline__ bool whole() const { return tiles == ntiles; }
    // committed tiles come first, the tree's is the last
    __device__ __forceinline__ bool is_tree(int tile) const { return t0 + tile == ntiles - 1; }
    __device__ __forceinline__ int valid(int T, int tile) const { return is_tree(tile) ? T : min(kTileKeys, L - (t0 + tile) * kTileKeys); }
    // A wide unit's steps are its tiles for slot 0 and for slot 1, in turn; a narrow one's are its tiles, in the slots in turn.
    __device__ __forceinline__ int steps() const { return wide ? 2 * tiles : tiles; }
    __device__ __forceinline__ int tile_of(int step) const { return wide ? step >> 1 : step; }
};
// The n-th use of the ring: its slot, and the parity of the slot's use.
struct Place {
    int s, parity;
    __device__ __forceinline__ Place(int n, bool six) {
        const int q = (unsigned)n / kRawSlots, r = n - q * kRawSlots;
        s = six ? r + (q & 1) * kRawSlots : r;
        parity = (six ? q >> 1 : q) & 1;
    }
};
struct Bars {
    // A slot has a barrier for each group of unpacking warps.  (The groups have its uses in turns, and a parity tells a phase only from the one before: at a common barrier a
    // group would take a use of the other's that is still on its way for its own.  Copies need not come in order.)
    uint64_t raw_full[2][2 * kRawSlots], raw_empty[2 * kRawSlots], k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t q_full, q_empty, s_full[2], p_full[2], pv_done, o_full, piece_full[kAhead], piece_empty[kAhead];
    uint32_t tmem_base;
    int32_t abort;
    int32_t raw_bad[2 * kRawSlots];   // a page outside the pool among the slot's
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
    uint32_t at = raw + scales_at(D) + (g * 4 + u / kPer) * 8 * kPer + j0 * kPer;
    uint32_t dst = tile + (w >> 3) * Cfg<D>::kBlock + (row0 + 8 * j0 + g) * 128 + (((w & 7) ^ g) << 4), src = raw + (8 * j0 + g) * (D / 2) + w * 4;
    const uint32_t odd = kPer == 2 ? (u & 1) * 0x0101u : 0u;
#pragma unroll 1
    for (int n = 0; n < 8 / kSplit; n += 4, at += 4 * kPer, src += 4 * 8 * (D / 2), dst += 4 * 8 * 128) {   // (all eight at once: more code than the instruction caches like)
        uint32_t codes[2] = {}, word[4];
        if constexpr (D == 128) { const uint2 x = lds64(at); codes[0] = x.x; codes[1] = x.y; }
        else codes[0] = lds32(at);
#pragma unroll
        for (int j = 0; j < 4; ++j) word[j] = lds32(src + j * 8 * (D / 2));
        auto go = [&](auto whole) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                constexpr bool kWhole = decltype(whole)::value;
                const uint32_t sel = 0x4040u | (j * kPer & 3) * 0x0101u;
                const Scale2 s = scale2<kWhole>(__byte_perm(codes[j * kPer >> 2], 0, sel + odd));
                sts128(dst + j * 8 * 128, pair<0>(word[j], s, sixteen), pair<1>(word[j], s, sixteen), pair<2>(word[j], s, sixteen), pair<3>(word[j], s, sixteen));
            }
        };
        if (nan_bits(codes[0]) | nan_bits(codes[1])) go(std::false_type());
        else go(std::true_type());
    }
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
    const uint32_t rows = page + (z * (D / 8) + f * (D / 16)) * 128;
#pragma unroll 1
    for (int y = 0; y < kWords; ++y) {
        // row d = z D/8 + f D/16 + 4 y + i
        const int turn = 4 * y + (D == 128 ? 0 : 4 * f);   // (of the row's number, what its place in the swizzle goes by)
        auto row = [&](int i) { return rows + (4 * y + i) * 128 + ((q ^ (turn + i)) << 4); };
        sts128(row(0), pair<0>(w[0][0], s[0], sixteen), pair<0>(w[1][0], s[1], sixteen), pair<0>(w[2][0], s[2], sixteen), pair<0>(w[3][0], s[3], sixteen));
        sts128(row(1), pair<1>(w[0][0], s[0], sixteen), pair<1>(w[1][0], s[1], sixteen), pair<1>(w[2][0], s[2], sixteen), pair<1>(w[3][0], s[3], sixteen));
        sts128(row(2), pair<2>(w[0][0], s[0], sixteen), pair<2>(w[1][0], s[1], sixteen), pair<2>(w[2][0], s[2], sixteen), pair<2>(w[3][0], s[3], sixteen));
        sts128(row(3), pair<3>(w[0][0], s[0], sixteen), pair<3>(w[1][0], s[1], sixteen), pair<3>(w[2][0], s[2], sixteen), pair<3>(w[3][0], s[3], sixteen));
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k][0] = w[k][kWords - 1];
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
        for (int i = 0; i < 2 * kRawSlots; ++i) {
            mbar_init(bar(&m->raw_full[0][i]), 1);
            mbar_init(bar(&m->raw_full[1][i]), 1);
            mbar_init(bar(&m->raw_empty[i]), kUnpackWarps);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&m->k_full[i]), kUnpackWarps);
            mbar_init(bar(&m->k_empty[i]), 1);
            mbar_init(bar(&m->v_full[i]), kUnpackWarps);
            mbar_init(bar(&m->v_empty[i]), 1);
            mbar_init(bar(&m->s_full[i]), 1);
            mbar_init(bar(&m->p_full[i]), kSoftmaxThreads / 32);
        }
        m->task.first = -1;
        mbar_init(bar(&m->q_full), 1);
        mbar_init(bar(&m->q_empty), 1);
        mbar_init(bar(&m->pv_done), 1);
        mbar_init(bar(&m->o_full), 1);
        for (int i = 0; i < kAhead; ++i) {
            mbar_init(bar(&m->piece_full[i]), 1);
            mbar_init(bar(&m->piece_empty[i]), kReaders);
            m->flags[i] = m->poison[i] = 0;
        }
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
    const bool six = list.n_wide == 0;   // slots of the ring

    if (warp >= kLoadWarp) {
        regs_dec<kRegsRest>();
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
            int n = 0, tiles = 0;                // slots of the ring, tiles so far
            uint32_t parity = 0, of_group = 0;   // bit slot + 8 group: of the next use; bit slot: whose the last use is
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
                        const Place slot(n, six);
                        if (!wait(bar(&m->raw_empty[slot.s]), slot.parity ^ 1, abort_s)) break;
                        if (lane == 0) {
                            m->raw_bad[slot.s] = !(ok0 && ok1);
                            const uint32_t full = bar(&m->raw_full[(tiles + t) & 1][slot.s]), dst = base + C::raw_at(slot.s);
                            const unsigned char *pool = kv ? p.v_pool : p.k_pool;
                            const int bytes = (ok0 ? C::kPageBytes : 0) + (count == 2 && ok1 ? C::kPageBytes : 0);
                            mbar_arrive_expect_tx(full, bytes);   // (a page outside the pool is not read; what the slot holds is never shown)
                            if (ok0) bulk_load(dst, pool + ((size_t)id0 * p.Hkv + x.h) * C::kPageBytes, C::kPageBytes, full, policy, streamed);
                            if (count == 2 && ok1) bulk_load(dst + C::kPageBytes, pool + ((size_t)id1 * p.Hkv + x.h) * C::kPageBytes, C::kPageBytes, full, policy, streamed);
                        }
                        __syncwarp();
                        parity ^= 1u << (slot.s + 8 * ((tiles + t) & 1));
                        of_group = (of_group & ~(1u << slot.s)) | ((tiles + t) & 1u) << slot.s;
                    }
                }
                tiles += x.tiles;
            }
            if (gone(abort_s)) {   // the block does not end under its own copies
                const uint64_t t0 = globaltimer_ns();
                for (int i = max(0, n - (six ? 2 : 1) * kRawSlots); i < n; ++i) {
                    const int s = Place(i, six).s, group = (of_group >> s) & 1;
                    while (!mbar_try_wait(bar(&m->raw_full[group][s]), ((parity >> (s + 8 * group)) & 1) ^ 1) && globaltimer_ns() - t0 < 20000000ull) {
                    }
                }
            }
        } else if (warp == kQueryWarp) {
            // ------------------------------------------------------------------ queries
            // A wide unit's rows fill both halves of the place, a narrow one's the first.  A unit has it when the one before is done with its last scores: while
            // that one's last probabilities and results are under way.
            constexpr int kChunks = D / 8, kRowsAtOnce = 32 / kChunks;
            const int ch = lane % kChunks, r0 = lane / kChunks;
            Piece x;
            for (int seg = 0; next_piece(m, x, seg, lane, abort_s); ++seg) {
                if (seg > 0) wait(bar(&m->q_empty), (seg - 1) & 1, abort_s);
                // row r of the head: of node g / G, (j Hq + h G + g - j G) D elements behind the sequence's first
                const __nv_bfloat16 *src = p.q + ((size_t)x.b * p.T * p.Hq + x.h * p.G) * D + ch * 8;
                uint32_t dst = base + C::kOffQ + (ch >> 3) * C::kBlock + r0 * 128;
                for (int r = r0; r < (x.wide ? 256 : 128); r += 8, dst += 8 * 128) {
                    if (r == 128 + r0) dst += C::kQBytes - C::kBlock;
#pragma unroll
                    for (int i = 0; i < 8; i += kRowsAtOnce) {
                        const bool live = r + i < x.rows;
                        const int g = x.rt * 256 + (live ? r + i : 0);
                        const __nv_bfloat16 *at = src + (size_t)(unsigned)(node_of(p, g) * (p.Hq - p.G) + g) * D;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + i * 128 + (((ch & 7) ^ (r0 + i)) << 4)), "l"(at), "r"(live ? 16 : 0) : "memory");
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&m->q_full));
            }
        } else {
            // ------------------------------------------------------------------ products
            constexpr uint32_t kIdescQK = idesc_bf16_f32(128, kTileKeys, false, false), kIdescPV = idesc_bf16_f32(128, D, false, false);
            const uint64_t descQ = smem_desc_sw128(base + C::kOffQ, 16, 1024), descK = smem_desc_sw128(base + C::kOffK, 16, 1024);
            const uint64_t descV = smem_desc_sw128(base + C::kOffV, 16, 1024);
            int nk = 0, nv = 0;          // tiles of keys, of values so far
            uint32_t p_parity = 0;       // bit `slot`
            Piece x;
            for (int seg = 0; next_piece(m, x, seg, lane, abort_s); ++seg) {
                wait(bar(&m->q_full), seg & 1, abort_s);
                const int steps = x.steps();
                auto score = [&](int i) {
                    const int slot = i & 1;
                    if (!x.wide || slot == 0) {
                        wait(bar(&m->k_full[nk & 1]), (nk >> 1) & 1, abort_s);
                        ++nk;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        const int buf = (nk - 1) & 1;
                        const uint64_t kd = descK + (uint64_t)((buf * C::kKBytes) >> 4), qd = descQ + (uint64_t)(((x.wide ? slot : 0) * C::kQBytes) >> 4);
                        const uint32_t tS = tmem + kTmemS + slot * 128;
#pragma unroll
                        for (int hf = 0; hf < C::kHalves; ++hf)
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                mma_bf16_ss(tS, qd + (uint64_t)((hf * C::kBlock + kk * 32) >> 4), kd + (uint64_t)((hf * C::kBlock + kk * 32) >> 4), kIdescQK, (hf | kk) != 0);
                        mma_commit(bar(&m->s_full[slot]));
                        if (!x.wide || slot == 1) mma_commit(bar(&m->k_empty[buf]));
                        if (i == steps - 1) mma_commit(bar(&m->q_empty));
                    }
                    __syncwarp();
                };
#pragma unroll 1
                for (int i = -2; i < steps; ++i) {
                    if (i >= 0) {
                        const int slot = i & 1, slices = (x.valid(p.T, x.tile_of(i)) + 15) >> 4;
                        if (!x.wide || slot == 0) {
                            wait(bar(&m->v_full[nv & 1]), (nv >> 1) & 1, abort_s);
                            ++nv;
                        }
                        wait(bar(&m->p_full[slot]), (p_parity >> slot) & 1, abort_s);
                        p_parity ^= 1u << slot;
                        tc_fence_after();
                        if (elect_one()) {
                            const int buf = (nv - 1) & 1;
                            const uint64_t vd = descV + (uint64_t)((buf * C::kVBytes) >> 4);
                            const uint32_t tP = tmem + kTmemS + slot * 128, tO = tmem + kTmemO + (x.wide ? slot * D : 0);
                            const bool fresh = x.tile_of(i) == 0;
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)   // (P of the keys 64 .. 127 lies over their scores)
                                if (kk < slices)
                                    mma_bf16_ts(tO, tP + (kk >> 2) * 64 + (kk & 3) * 8, vd + (uint64_t)(((kk >> 2) * C::kVPage + (kk & 3) * 32) >> 4), kIdescPV, !fresh || kk != 0);
                            if (!x.wide || slot == 1) mma_commit(bar(&m->v_empty[buf]));
                            if (i == steps - 1) mma_commit(bar(&m->o_full));
                            if (!x.wide) mma_commit(bar(&m->pv_done));
                        }
                        __syncwarp();
                    }
                    if (i + 2 < steps) score(i + 2);
                }
            }
            if (gone(abort_s)) __nanosleep(1000000);   // products that are still under way end before their operands go away
        }
    } else if (warp >= kUnpackWarp) {
        // ------------------------------------------------------------------ unpacking
        regs_dec<kRegsUnpack>();
        const int group = (warp - kUnpackWarp) >> 2, t = tid & 127;   // the groups of four warps unpack every other tile
        volatile uint32_t *word = reinterpret_cast<volatile uint32_t *>(smem + C::kOffSwap);   // (an opaque constant: see pair())
        if (t == 0) *word = 0x41804180u;
        asm volatile("bar.sync 2, 256;" ::: "memory");
        const uint32_t sixteen = *word;
        asm volatile("bar.sync 2, 256;" ::: "memory");
        int n = 0, raw = 0, trees = 0;   // tiles, slots of the ring, trees so far
        uint32_t parity = 0;             // bit slot: of the group's next use
        Piece x;
        for (int seg = 0; next_piece(m, x, seg, lane, abort_s); ++seg) {
            const bool has_tree = x.is_tree(x.tiles - 1);
            for (int i = (n ^ group) & 1; i < x.tiles; i += 2) {
                const uint32_t kt = base + C::kOffK + group * C::kKBytes, vt = base + C::kOffV + group * C::kVBytes;
                const uint32_t free = (((n + i) >> 1) & 1) ^ 1;
                const bool tree = has_tree && i == x.tiles - 1;
                const int valid = x.valid(p.T, i);
                // keys
                if (!wait(bar(&m->k_empty[group]), free, abort_s)) break;
                if (tree) {
                    unsigned char *parents = smem + C::kOffParents + (trees & (kAhead / 2 - 1)) * kMaxNodes;
                    if (t < p.T) {
                        const int a = p.parent[(size_t)x.b * p.T + t];
                        parents[t] = (unsigned char)a;
                        if (!(t == 0 ? a == -1 : a >= 0 && a < t)) atomicOr(&m->flags[seg & (kAhead - 1)], kBadTree);
                    }
                    copy_tree_keys<D>(p, x.b, x.h, kt, t);
                } else {
                    const Place at(raw + 2 * i, six);
                    if (!wait(bar(&m->raw_full[group][at.s]), (parity >> at.s) & 1, abort_s)) break;
                    parity ^= 1u << at.s;
                    const uint32_t src = base + C::raw_at(at.s);
                    if (m->raw_bad[at.s] && t == 0) atomicOr(&m->flags[seg & (kAhead - 1)], kBadPage);
#pragma unroll 1
                    for (int page = 0; page * kPage < valid && page < 2; ++page) unpack_keys<D>(src + page * C::kPageBytes, kt, page * kPage, t, sixteen);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&m->raw_empty[at.s]));
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&m->k_full[group]));
                // values
                if (!wait(bar(&m->v_empty[group]), free, abort_s)) break;
                if (tree) {
                    if (copy_tree_values<D>(p, x.b, x.h, vt, t)) atomicOr(&m->poison[seg & (kAhead - 1)], 1);
                } else {
                    const Place at(raw + 2 * i + 1, six);
                    if (!wait(bar(&m->raw_full[group][at.s]), (parity >> at.s) & 1, abort_s)) break;
                    parity ^= 1u << at.s;
                    const uint32_t src = base + C::raw_at(at.s);
#pragma unroll 1
                    for (int page = 0; page * kPage < valid && page < 2; ++page)
                        unpack_values<D>(src + page * C::kPageBytes, vt + page * C::kVPage, min(valid - page * kPage, kPage), t, sixteen);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&m->raw_empty[at.s]));
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&m->v_full[group]));
            }
            n += x.tiles;
            raw += 2 * (x.tiles - has_tree);
            trees += has_tree;
        }
    } else {
        // ------------------------------------------------------------------ softmax, results
        regs_inc<kRegsSoftmax>();
        // Two threads to a row, of warps `half` = 0 and 1: keys 64 half .. + 63 of a tile.
        const int half = warp >> 2, row = tid & 127;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        constexpr uint32_t kNegInf = 0xff800000u;
        float *top_s = reinterpret_cast<float *>(smem + C::kOffSwap), *sum_s = top_s + 256;
        const float by = raise_by(p);
        auto pair_barrier = [&]() { asm volatile("barrier.cta.sync %0, 64;" ::"r"(5 + (warp & 3)) : "memory"); };
        uint32_t s_parity = 0;   // bit `slot`
        uint32_t narrow_steps = 0;
        int trees = 0;
        // Whether there is another unit is decided together: a block that gives up may do so between two warps' looks at the ring, and the
        // barriers among the softmax threads want all of them.
        auto next_for_all = [&](Piece &y, int seg) {
            const bool got = next_piece(m, y, seg, lane, abort_s);
            int all;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 256, p;\n\tselp.b32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"((int)got) : "memory");
            return all != 0;
        };
        Piece x;
        for (int seg = 0; next_for_all(x, seg); ++seg) {
            // A row without a query never asks for a higher maximum.  (m, l) of the step's slot, and of the other (wide)
            const int r_end = x.rows;
            float mx = row < r_end ? -INFINITY : INFINITY, l = 0.f, mx_other = 128 + row < r_end ? -INFINITY : INFINITY, l_other = 0.f;
            const bool has_tree = x.is_tree(x.tiles - 1);
            const int steps = x.steps();
#pragma unroll 1
            for (int i = 0; i < steps; ++i) {
                const int slot = i & 1, t = x.tile_of(i), r = (x.wide ? slot * 128 : 0) + row;
                const uint32_t tS = tmem + kTmemS + slot * 128 + half * 64 + lane_base;
                const bool live = r < r_end, warp_live = __any_sync(0xffffffffu, live);
                wait(bar(&m->s_full[slot]), (s_parity >> slot) & 1, abort_s);
                s_parity ^= 1u << slot;
                tc_fence_after();
                if (warp_live) {
                    const int valid = x.valid(p.T, t) - half * 64;   // of this half's keys
                    if (valid < 64 || x.is_tree(t)) {                // scores of keys that a row does not see become -inf
                        uint64_t sees = ~0ull;
                        if (x.is_tree(t)) {
                            const int g = x.rt * 256 + r, node = live ? node_of(p, g) : 0;
                            sees = 0;
                            if (live && p.anc) {
                                sees = p.anc[((size_t)x.b * p.T + node) * 2 + half];
                            } else if (live && !(*(volatile int32_t *)&m->flags[seg % kAhead] & kBadTree)) {
                                const unsigned char *parents = smem + C::kOffParents + (trees & (kAhead / 2 - 1)) * kMaxNodes;
                                sees = ancestors(parents, node, half);
                            }
                        }
                        if (valid < 64) sees &= valid <= 0 ? 0 : (1ull << valid) - 1;
#pragma unroll 1
                        for (int c = 0; c < 64; c += 16, sees >>= 16) {
                            uint32_t y[16];
                            tmem_ld16(tS + c, y);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                if (!((sees >> k) & 1)) y[k] = kNegInf;
                            tmem_st16(tS + c, y);
                        }
                        tmem_wait_st();
                    }
                    // Half of the scores at a time, the second ones first, so that the first are at hand for what follows
                    uint32_t s[32];
                    auto f = [&](int k) { return __uint_as_float(s[k]); };
                    float top = -INFINITY;
#pragma unroll 1
                    for (int c = 32; c >= 0; c -= 32) {
                        tmem_ld32(tS + c, s);
                        tmem_wait_ld();
                        float a[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) a[k] = max3(f(8 * k), f(8 * k + 1), f(8 * k + 2));
#pragma unroll
                        for (int i = 3; i < 7; i += 2)
#pragma unroll
                            for (int k = 0; k < 4; ++k) a[k] = max3(a[k], f(8 * k + i), f(8 * k + i + 1));
#pragma unroll
                        for (int k = 0; k < 4; ++k) a[k] = fmaxf(a[k], f(8 * k + 7));
                        top = max3(max3(top, a[0], a[1]), a[2], a[3]);
                    }
                    int raise;
                    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.gt.f32 p, %1, %2;\n\tbarrier.cta.red.or.pred q, %3, 64, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                                 : "=r"(raise) : "f"(top), "f"(mx + by), "r"(5 + (warp & 3)) : "memory");
                    if (raise) {
                        top_s[half * 128 + row] = top;
                        pair_barrier();
                        const float now = max3(mx, top, top_s[(half ^ 1) * 128 + row]);
                        const float g = mx == now ? 1.f : ex2((mx - now) * p.scale_log2);   // (-inf before the first score: 0)
                        mx = now;
                        l *= g;
                        if (t > 0) {
                            // A wide unit's products of this slot are done, these scores having come behind them; a narrow one's last are awaited.
                            if (!x.wide) {
                                wait(bar(&m->pv_done), (narrow_steps - 1) & 1, abort_s);
                                tc_fence_after();
                            }
                            const uint32_t tO = tmem + kTmemO + (x.wide ? slot * D : 0) + half * (D / 2) + lane_base;
#pragma unroll 1
                            for (int c = 0; c < D / 2; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(tO + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * g);
                                tmem_st16(tO + c, o);
                            }
                        }
                    }
                    // 2^((s - max) scale) by one multiplication and addition.  The maximum times the scale is rounded, by the same for all keys that are weighed with
                    // this maximum, among which that cancels; between steps and shares with other maxima it does not, and is 2^-24 of the scaled maximum at most, as
                    // fp32 scores of that size themselves are: up to 65536, 2^-9 or 0.14 % of a weight, a third of what a probability's rounding to bf16 may be.
                    // Beyond that, or beyond fp32, the difference is taken first.  (A row without a query, and one with an infinite score, has an infinite maximum: no
                    // difference helps.)
                    float from = mx == -INFINITY ? 0.f : -mx * p.scale_log2;
                    if (__any_sync(0xffffffffu, fabsf(from) > 65536.f && fabsf(mx) < INFINITY)) {
#pragma unroll 1
                        for (int c = 0; c < 64; c += 16) {
                            uint32_t y[16];
                            tmem_ld16(tS + c, y);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) - (mx == -INFINITY ? 0.f : mx));
                            tmem_st16(tS + c, y);
                        }
                        tmem_wait_st();
                        tmem_ld32(tS, s);
                        tmem_wait_ld();
                        from = 0.f;
                    }
                    const float2 from2 = make_float2(from, from), sc = make_float2(p.scale_log2, p.scale_log2);
                    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 1
                    for (int c = 0; c < 32; c += 16) {   // (probabilities over scores that have been read)
                        uint32_t pk[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            const float2 y = __ffma2_rn(make_float2(f(2 * k), f(2 * k + 1)), sc, from2);
                            const float2 e = make_float2(ex2(y.x), ex2(y.y));
                            sum = __fadd2_rn(sum, e);
                            pk[k] = pack(e.x, e.y);
                        }
                        tmem_st16(tS + c, pk);
                        if (c == 0) {
                            tmem_ld32(tS + 32, s);
                            tmem_wait_ld();
                        }
                    }
                    l += sum.x + sum.y;
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&m->p_full[slot]));
                if (x.wide) {
                    const float a = mx, b = l;
                    mx = mx_other; l = l_other;
                    mx_other = a; l_other = b;
                } else ++narrow_steps;
            }
            // Results: a wide unit's slot `half`; of a narrow one half of the columns.
            wait(bar(&m->o_full), seg & 1, abort_s);
            tc_fence_after();
            const int r = (x.wide ? half * 128 : 0) + row, grow = x.rt * 256 + r;   // among the unit's rows, the head's
            const bool live = r < r_end, warp_live = __any_sync(0xffffffffu, live);
            const int node = live ? node_of(p, grow) : 0;
            const bool swap = x.wide && half == 1;
            sum_s[half * 128 + row] = x.wide && half == 0 ? l_other : l;
            softmax_barrier();
            mx = swap ? mx_other : mx;
            l = (swap ? l_other : l) + sum_s[(half ^ 1) * 128 + row];
            const int col0 = x.wide ? 0 : half * (D / 2), col1 = x.wide ? D : col0 + D / 2;
            const uint32_t tO = tmem + kTmemO + (x.wide ? half * D : 0) + lane_base;
            int flag = *(volatile int32_t *)&m->flags[seg % kAhead];
            if (*abort_s || (int)blockIdx.x == p.give_up) flag |= kGaveUp;
            if (has_tree && *(volatile int32_t *)&m->poison[seg % kAhead] && warp_live && !(flag & kBadTree)) {
                // Infinities and NaN were left out of the product: the rows that see them get them.  All nodes' before the columns are stored again: a store to tensor
                // memory is not there for the next load until it has been waited for.
                uint64_t sees0 = 0, sees1 = 0;
                if (live && p.anc) {
                    sees0 = p.anc[((size_t)x.b * p.T + node) * 2];
                    sees1 = p.anc[((size_t)x.b * p.T + node) * 2 + 1];
                } else if (live) {
                    sees0 = ancestors(p.parent + (size_t)x.b * p.T, node, 0);
                    sees1 = ancestors(p.parent + (size_t)x.b * p.T, node, 1);
                }
                const uint32_t *val = reinterpret_cast<const uint32_t *>(p.v_tree + ((size_t)x.b * p.T * p.Hkv + x.h) * D);
#pragma unroll 1
                for (int c = col0; c < col1; c += 16) {
                    uint32_t o[16];
                    tmem_ld16(tO + c, o);
                    tmem_wait_ld();
#pragma unroll 1
                    for (int n = 0; n < p.T; ++n) {
                        if (!(((n < 64 ? sees0 : sees1) >> (n & 63)) & 1)) continue;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const uint32_t w = val[(size_t)n * p.Hkv * (D / 2) + c / 2 + i];
                            if (nonfinite(w << 16)) o[2 * i] = __float_as_uint(__uint_as_float(o[2 * i]) + bf16lo(w));
                            if (nonfinite(w)) o[2 * i + 1] = __float_as_uint(__uint_as_float(o[2 * i + 1]) + bf16hi(w));
                        }
                    }
                    __syncwarp();
                    tmem_st16(tO + c, o);
                }
                tmem_wait_st();
            }
            const size_t orow = ((size_t)x.b * p.T + node) * p.Hq + x.h * p.G + (grow - node * p.G);
            const int share = 2 * blockIdx.x + (x.t0 == 0 ? 1 : 0);
            const size_t srow = (size_t)share * 256 + r;
            const float inv = flag || l == 0.f ? 0.f : 1.f / l;   // (a row that sees nothing: zeros)
            if (warp_live) {
#pragma unroll 1
                for (int c = col0; c < col1; c += 16) {
                    uint32_t o[16];
                    tmem_ld16(tO + c, o);
                    tmem_wait_ld();
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
                        uint4 *dst = reinterpret_cast<uint4 *>(p.partial_o) + (size_t)share * 256 * (D / 4) + (c / 4) * 256 + r;   // [D / 4][rows]: neighbouring threads' together
#pragma unroll
                        for (int i = 0; i < 4; ++i) dst[i * 256] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                }
                if (live && (x.wide || half == 0)) {
                    if (!x.whole()) p.partial_ml[srow] = make_float2(mx, l);
                    else if (p.lse) p.lse[orow] = flag ? 0.f : fmaf(mx, p.scale, log2f(l) * 0.6931471805599453f);
                }
            }
            tc_fence_before();
            softmax_barrier();   // all have read the flags
            if (tid == 0) {
                m->flags[seg % kAhead] = 0;
                m->poison[seg % kAhead] = 0;
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

// Units that several blocks have shares of: eight rows of the one that block blockIdx.x of the attention begins, a thread to four elements of a row.
// (A launch of its own: the block that came last did this at first, and took 25 us for the shares of 128 rows and 60 us for those of 256,
// the others waiting.)
template <int D>
__global__ void __launch_bounds__(2 * D) q4_attn_merge_kernel(const __grid_constant__ Q4AttnParams p) {
    const int r = blockIdx.y * 8 + (threadIdx.x & 7), c = threadIdx.x >> 3;
    pdl_wait();
    pdl_launch_dependents();
    const ShareTask t = p.tasks[blockIdx.x];
    if (t.first < 0 || r >= t.rows) return;
    const Part y = merge_shares(p, t, 0, t.last - t.first + 1, 256, r, [&](int share) { return reinterpret_cast<const float4 *>(p.partial_o)[(size_t)share * 256 * (D / 4) + c * 256 + r]; });
    put_merged<D>(p, t, 256, r, c, y);
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
    launch_q4_attn_status(p, st);
    launch_pdl(p.D == 128 ? q4_attn_sm100_kernel<128> : q4_attn_sm100_kernel<64>, dim3((unsigned)n_sm), dim3(kThreads),
               (size_t)(p.D == 128 ? Cfg<128>::kSmem : Cfg<64>::kSmem), st, p);
    launch_pdl(p.D == 128 ? q4_attn_merge_kernel<128> : q4_attn_merge_kernel<64>, dim3((unsigned)n_sm, (unsigned)((std::min(256, p.T * p.G) + 7) / 8)), dim3(2 * p.D), 0,
               st, p);
    return READER_OK;
}

}  // namespace reader

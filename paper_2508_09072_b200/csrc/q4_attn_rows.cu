// Tree-masked attention over a 4-bit cache for few query rows (reader_q4_verify_attn): single tokens, small trees.
//
// A unit is (sequence, KV head, 8 or 16 query rows).  Bound: bytes, 72 D of every 64 positions and head, if the numbers become
// operands fast enough.  So they never leave a warp: each warp is a worker of its own that brings tiles (one page of keys or
// values of one head, 36 D bytes) into its own ring in shared memory by bulk copies and computes S^T = K Q^T and O^T += V^T P^T with
// m16n8k16 products: keys and values are the 16-row operand, query rows the 8-column one, so that a row of queries costs
// nothing that is not its own.  The A fragments are unpacked in registers, two bf16 in 2.75 instructions; the pages are laid
// out so that a lane's words, and their scales, are one or two 16-byte loads.  (Feeding tcgen05.mma instead means writing every
// tile in bf16 to shared memory and reading it back: worth it once many rows share it, not for 4 or 16.)  Measured (32 query heads, 8 KV heads, head_dim 128):
// single tokens on 32 contexts of 1024-4096 34 us, 0.44 of the copy bandwidth, 25 to 28 of them the walk; on 64 of 2048-8192 87 us, 0.68;
// one token on 511 (8 heads, head_dim 64) 6.1 us.  A product's inner order
// is free as long as both operands agree: of the elements, lane (g, c) = (lane / 4, lane % 4) has D/4 consecutive ones of a key,
// and D/8 consecutive ones of a pair of values, with one or two scales; P^T gets from the score product's result to the value
// product's operand by one transposing move per 8 x 8 block.
//
// Two forms.  (Alone) A call with few units is one launch: a cluster of thread blocks per unit, whose workers share its
// tiles; shares (m, l, O) are merged in shared memory, those of the cluster's blocks through the workspace after its barrier.
// (List) The units, each preceded by kUnitCost entries for its start and end, form one flat list of tiles that is cut into equal
// ranges, one per worker, those of a thread block side by side.  Every thread block makes the list's prefix sums from seq_lens
// itself.  A worker writes a unit that lies in its range whole, and leaves a share (m, l, O) of any other in the workspace; a launch behind merges them.
// (The blocks did it themselves at first, in shared memory, and then the one that came last: 9 us of a call over 32 contexts of 1024-4096 for 4 rows,
// 24 us for 16.)
//
// What is checked where: lengths by every block, page ids by the worker that reads them, a tree by the worker of the unit's
// tree tiles; what is wrong travels with the share and zeroes the unit's rows.  Bytes behind a sequence's end never reach a
// product: their scores are replaced by -inf and their values' scale by 0.  Every wait is bounded; a worker that gives up says so
// in its share, waits (bounded) for its copies and goes on without them.
#include <algorithm>

#include "q4_attn_common.cuh"

namespace reader {
namespace {

using namespace q4;

// Workers of a thread block, and their ring's slots (a tile of keys or of values each): what registers and shared memory allow.  At head_dim 128 registers do not
// quite: of 128 to a thread the list form's kernel for 8 rows spills 36 bytes (64 read back), of 168 that for 16 rows 208 (272); the form of one launch 8 (16) and
// 88 (152).
template <int NT>
struct Shape {
    static constexpr int kWarps = NT == 1 ? 16 : 12, kSlots = NT == 1 ? 3 : 4;
    static constexpr int kThreads = kWarps * 32, kRows = 8 * NT;
};
constexpr int kUnitCost = 2;       // entries that stand for a unit's start and end
constexpr int kMinEntries = kUnitCost + 1;   // of a range: so every one of them holds a tile

template <int D, int NT>
struct Cfg {
    using S = Shape<NT>;
    static constexpr int kTile = q4::tile_bytes(D);
    static constexpr int kRingBytes = S::kSlots * kTile;   // of one worker; its share (rows x D floats) when all is done
    static constexpr int kOffBars = S::kWarps * kRingBytes;
    static constexpr int kOffParents = kOffBars + S::kWarps * S::kSlots * 8;
    static constexpr int kOffMasks = kOffParents + S::kWarps * kMaxNodes;
    static constexpr int kOffShares = kOffMasks + S::kWarps * S::kRows * 16;           // (m, l) of the workers' rows
    static constexpr int kOffPrefix = kOffShares + S::kWarps * S::kRows * 8;           // first entry, length of each sequence
    static constexpr int kSmem = kOffPrefix + kPrefix * 8;
    static_assert(kSmem + 1024 <= 227 * 1024 && kRingBytes >= S::kRows * D * 4, "shared memory");
};

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transposed 8 x 8 block of 16-bit elements: lane (g, c) gives elements (g, 2 c), (g, 2 c + 1) and gets (2 c, g), (2 c + 1, g).
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// ---- rows of a unit
template <int NT>
__device__ __forceinline__ size_t out_row(const Q4AttnParams &p, int b, int h, int rt, int r) {
    const int row = rt * Shape<NT>::kRows + r, j = node_of(p, row);
    return ((size_t)b * p.T + j) * p.Hq + h * p.G + (row - j * p.G);
}
template <int NT>
__device__ __forceinline__ int live_rows(const Q4AttnParams &p, int rt) { return min(Shape<NT>::kRows, p.T * p.G - rt * Shape<NT>::kRows); }
// ---- one worker
template <int D, int NT>
struct Worker {
    using S = Shape<NT>;
    using C = Cfg<D, NT>;
    static constexpr int kSteps = D / 16;    // inner steps of the score product, 16-row tiles of the value product
    static constexpr int kOwn = D / 8;       // value elements of a lane
    const Q4AttnParams &p;
    uint32_t ring, bars;
    uint32_t sixteen;        // 16 in bf16, twice; in a register of its own (a second constant in the instruction cannot be)
    int lane, g, c;
    int issued, used;        // tiles of keys or values, counted over the worker's life
    bool gave_up;
    // the unit's page ids, 32 at a time
    int ids, ids_next, ids_at, t_issue;

    uint32_t qf[kSteps][NT][2];
    float o[kSteps][NT][4];   // O^T: elements 16 g' .. of rows 2 c, 2 c + 1 of each 8
    float m[NT][2], l[NT][2]; // rows 2 c, 2 c + 1; l: this lane's share

    __device__ __forceinline__ Worker(const Q4AttnParams &p_) : p(p_) {}

    __device__ __forceinline__ void init(unsigned char *smem, int warp) {
        lane = threadIdx.x & 31; g = lane >> 2; c = lane & 3;
        const uint32_t base = smem_u32(smem);
        ring = base + warp * C::kRingBytes;
        bars = base + C::kOffBars + warp * S::kSlots * 8;
        issued = used = 0;
        gave_up = false;
        volatile uint32_t *word = reinterpret_cast<volatile uint32_t *>(smem + warp * C::kRingBytes);
        if (lane == 0) {
            *word = 0x41804180u;
            for (int s = 0; s < S::kSlots; ++s) mbar_init(bars + s * 8, 1);
            fence_mbar_init();
        }
        __syncwarp();
        sixteen = *word;
        __syncwarp();
        fence_proxy_async();
    }

    // ---- tiles
    __device__ __forceinline__ int page_ids(const Unit &u, int t, int &flag) {
        const int pages_end = min(u.t1, u.npages);
        int id = 0;
        if (t + lane < pages_end) {
            id = p.page_table[(size_t)u.b * p.max_pages + t + lane];
            if (id < 0 || id >= p.num_pages) {
                flag |= kBadPage;
                id = 0;
            }
        }
        return id;
    }
    // The next tile of the unit: keys of page t, values of page t, keys of page t + 1, ...
    __device__ __forceinline__ void issue(const Unit &u, uint64_t policy, bool once, int &flag) {
        const int t = t_issue >> 1;
        if (t - ids_at == 32) {
            ids_at = t;
            ids = ids_next;
            ids_next = page_ids(u, t + 32, flag);
        }
        const int page = __shfl_sync(0xffffffffu, ids, t - ids_at);
        if (lane == 0) {
            const int s = issued % S::kSlots;
            const uint32_t bar = bars + s * 8;
            mbar_arrive_expect_tx(bar, C::kTile);
            bulk_load(ring + s * C::kTile, ((t_issue & 1) ? p.v_pool : p.k_pool) + ((size_t)page * p.Hkv + u.h) * C::kTile, C::kTile, bar, policy,
                      once && t >= p.shared_prefix_pages);
        }
        ++issued;
        ++t_issue;
    }
    __device__ __forceinline__ void start(const Unit &u, int pages_end, uint64_t policy, bool once, int &flag) {
        ids_at = u.t0;
        t_issue = 2 * u.t0;
        ids = page_ids(u, u.t0, flag);
        ids_next = pages_end - u.t0 > 32 ? page_ids(u, u.t0 + 32, flag) : 0;
#pragma unroll 1
        for (int i = 0; i < S::kSlots && t_issue < 2 * pages_end; ++i) issue(u, policy, once, flag);
    }
    // The slot of the next tile once it is there.
    __device__ __forceinline__ uint32_t await() {
        const int s = used % S::kSlots;
        const uint32_t bar = bars + s * 8, parity = (used / S::kSlots) & 1;
        if (!mbar_try_wait(bar, parity)) {
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar, parity))
                if (globaltimer_ns() - t0 > kWaitLimitNs) {
                    gave_up = true;
                    break;
                }
        }
        gave_up = __any_sync(0xffffffffu, gave_up);
        return ring + s * C::kTile;
    }
    __device__ __forceinline__ void release() {
        ++used;
        __syncwarp();
    }

    // ---- queries: lane (g, c) has elements c D/4 .. of row g of each 8
    __device__ __forceinline__ void begin(const Unit &u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = u.rt * S::kRows + 8 * nt + g;
            const bool live = r < p.T * p.G;
            const int j = live ? node_of(p, r) : 0, hq = u.h * p.G + (live ? r - j * p.G : 0);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (((size_t)u.b * p.T + j) * p.Hq + hq) * D + c * (D / 4));
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                const uint4 v = live ? src[x] : make_uint4(0, 0, 0, 0);
                qf[2 * x][nt][0] = v.x; qf[2 * x][nt][1] = v.y;
                qf[2 * x + 1][nt][0] = v.z; qf[2 * x + 1][nt][1] = v.w;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[nt][e] = -INFINITY;
                l[nt][e] = 0.f;
            }
#pragma unroll
            for (int x = 0; x < kSteps; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[x][nt][i] = 0.f;
        }
    }

    // ---- softmax of 16 kM keys (keys g and g + 8 of each 16, rows 2 c and 2 c + 1 of each 8): probabilities in place
    template <int kM>
    __device__ __forceinline__ void softmax(float (&s)[kM][NT][4]) {
        float top[NT][2];
        bool rises = false;
        // the maximum in use is raised only when a score exceeds it by 2^8: the vote needs no exchange
        const float by = raise_by(p);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float t = fmaxf(s[0][nt][e], s[0][nt][2 + e]);
#pragma unroll
                for (int j = 1; j < kM; ++j) t = max3(t, s[j][nt][e], s[j][nt][2 + e]);
                top[nt][e] = t;
                rises |= t > m[nt][e] + by;
            }
        if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float t = top[nt][e];
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
                    const float now = fmaxf(m[nt][e], t);
                    const float f = m[nt][e] == now ? 1.f : ex2((m[nt][e] - now) * p.scale_log2);   // (-inf before the first score: 0)
                    m[nt][e] = now;
                    l[nt][e] *= f;
#pragma unroll
                    for (int x = 0; x < kSteps; ++x) {
                        o[x][nt][e] *= f;
                        o[x][nt][2 + e] *= f;
                    }
                }
        }
        // The difference to the maximum is taken before the scaling: whatever the scores' size, it is as exact as they are.
        const float2 sc = make_float2(p.scale_log2, p.scale_log2);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float2 from = make_float2(m[nt][0] == -INFINITY ? 0.f : -m[nt][0], m[nt][1] == -INFINITY ? 0.f : -m[nt][1]);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < kM; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float2 x = __fmul2_rn(__fadd2_rn(make_float2(s[j][nt][2 * k], s[j][nt][2 * k + 1]), from), sc);
                    const float2 y = make_float2(ex2(x.x), ex2(x.y));
                    s[j][nt][2 * k] = y.x;
                    s[j][nt][2 * k + 1] = y.y;
                    sum = __fadd2_rn(sum, y);
                }
            l[nt][0] += sum.x;
            l[nt][1] += sum.y;
        }
    }

    static __device__ __forceinline__ void load_words(uint32_t (&w)[D / 32], uint32_t at) {
        if constexpr (D == 128) {
            const uint4 x = lds128(at);
            w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        } else {
            const uint2 x = lds64(at);
            w[0] = x.x; w[1] = x.y;
        }
    }
    // Whether a tile (of keys or values) holds a block that reads as NaN.
    __device__ __forceinline__ bool holds_nan(uint32_t tile) const {
        uint32_t any;
        if (D == 128) {
            const uint4 a = lds128(tile + q4::scales_at(D) + lane * 16);
            any = nan_bits(a.x) | nan_bits(a.y) | nan_bits(a.z) | nan_bits(a.w);
        } else {
            const uint2 a = lds64(tile + q4::scales_at(D) + lane * 8);
            any = nan_bits(a.x) | nan_bits(a.y);
        }
        return __any_sync(0xffffffffu, any != 0);
    }

    static constexpr int kPart = NT == 1 ? 4 : 2;   // 16-key tiles that go through the softmax together

    // Scores of the 16 kPart keys from key 16 j0 on.  kWhole: all committed, no block that reads as NaN.
    template <bool kWhole>
    __device__ __forceinline__ void scores(uint32_t k, int j0, int valid, float (&s)[kPart][NT][4]) {
        constexpr int kPer = D / 64;   // scales of a lane and key
        const uint32_t row = k + g * (D / 2) + c * (D / 8), at = k + q4::scales_at(D) + lane * (8 * kPer) + j0 * 2 * kPer;
        uint32_t cw[2] = {};
        if constexpr (kPart * kPer == 8) { const uint4 x = lds128(at); scores_of<kWhole>(row, j0, valid, s, {x.x, x.y, x.z, x.w}); return; }
        if constexpr (kPart * kPer == 4) { const uint2 x = lds64(at); cw[0] = x.x; cw[1] = x.y; }
        if constexpr (kPart * kPer == 2) cw[0] = lds32(at);
        scores_of<kWhole>(row, j0, valid, s, {cw[0], cw[1], 0, 0});
    }
    struct Words4 {
        uint32_t w[4];
    };
    template <bool kWhole>
    __device__ __forceinline__ void scores_of(uint32_t row, int j0, int valid, float (&s)[kPart][NT][4], const Words4 &cw) {
        constexpr int kPer = D / 64;
#pragma unroll
        for (int j = 0; j < kPart; ++j) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j][nt][i] = 0.f;
            uint32_t wa[D / 32], wb[D / 32];   // keys 16 j + g and 16 j + 8 + g
            load_words(wa, row + (j0 + j) * (16 * D / 2));
            load_words(wb, row + (j0 + j) * (16 * D / 2) + 8 * D / 2);
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                // the code of block x / 2 of either key, twice
                const int ba = 2 * j * kPer + x / 2, bb = ba + kPer;
                const Scale2 sa = scale2<kWhole>(__byte_perm(cw.w[ba / 4], 0, 0x4040 | (ba % 4) | ((ba % 4) << 8)));
                const Scale2 sb = scale2<kWhole>(__byte_perm(cw.w[bb / 4], 0, 0x4040 | (bb % 4) | ((bb % 4) << 8)));
                {
                    const uint32_t a0 = pair<0>(wa[x], sa, sixteen), a1 = pair<0>(wb[x], sb, sixteen), a2 = pair<1>(wa[x], sa, sixteen), a3 = pair<1>(wb[x], sb, sixteen);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(s[j][nt], a0, a1, a2, a3, qf[2 * x][nt][0], qf[2 * x][nt][1]);
                }
                {
                    const uint32_t a0 = pair<2>(wa[x], sa, sixteen), a1 = pair<2>(wb[x], sb, sixteen), a2 = pair<3>(wa[x], sa, sixteen), a3 = pair<3>(wb[x], sb, sixteen);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(s[j][nt], a0, a1, a2, a3, qf[2 * x + 1][nt][0], qf[2 * x + 1][nt][1]);
                }
            }
            if (!kWhole) {
                const int key = 16 * (j0 + j) + g;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (key >= valid) s[j][nt][0] = s[j][nt][1] = -INFINITY;
                    if (key + 8 >= valid) s[j][nt][2] = s[j][nt][3] = -INFINITY;
                }
            }
        }
    }
    // O^T += V^T P^T of the same keys.
    template <bool kWhole>
    __device__ __forceinline__ void values(uint32_t v, int j0, int valid, const float (&s)[kPart][NT][4]) {
        // position pair 8 j + 4 e + c: row of D bytes; of its eight chunks the one with this lane's elements
        const uint32_t row = v + c * D + q4::v_chunk<D>(c, g) * (D / 8);
        const uint32_t at = v + q4::scales_at(D) + ((D == 128 ? g : g >> 1) * 4 + c) * 16 + j0 * 4;
#pragma unroll
        for (int j = 0; j < kPart; ++j) {
            uint32_t b[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                b[nt][0] = transposed(pack(s[j][nt][0], s[j][nt][1]));
                b[nt][1] = transposed(pack(s[j][nt][2], s[j][nt][3]));
            }
            const uint32_t cw = lds32(at + 4 * j);
            uint32_t w[2][D / 32];
            Scale2 sc[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                load_words(w[e], row + (2 * (j0 + j) + e) * (4 * D));
                sc[e] = scale2<kWhole>(__byte_perm(cw, 0, e ? 0x4342 : 0x4140));
                if (!kWhole) {   // positions behind the end: scale 0, whatever their code
                    const int key = 8 * (2 * (j0 + j) + e) + 2 * c;
                    if (key >= valid) { sc[e].s &= 0xffff0000u; sc[e].m24 &= 0xffff0000u; }
                    if (key + 1 >= valid) { sc[e].s &= 0xffffu; sc[e].m24 &= 0xffffu; }
                }
            }
#pragma unroll
            for (int y = 0; y < D / 32; ++y) {
                {
                    const uint32_t a0 = pair<0>(w[0][y], sc[0], sixteen), a1 = pair<1>(w[0][y], sc[0], sixteen), a2 = pair<0>(w[1][y], sc[1], sixteen), a3 = pair<1>(w[1][y], sc[1], sixteen);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(o[2 * y][nt], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                }
                {
                    const uint32_t a0 = pair<2>(w[0][y], sc[0], sixteen), a1 = pair<3>(w[0][y], sc[0], sixteen), a2 = pair<2>(w[1][y], sc[1], sixteen), a3 = pair<3>(w[1][y], sc[1], sixteen);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(o[2 * y + 1][nt], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                }
            }
        }
    }

    // ---- the unit's pages from t0 on
    __device__ __forceinline__ void walk(const Unit &u, int pages_end, uint64_t policy, bool once, int &flag) {
#pragma unroll 1
        for (int t = u.t0; t < pages_end; ++t) {
            const int valid = min(kPage, u.L - t * kPage);
            float s[kPart][NT][4];
            const uint32_t k = await();
            if (gave_up) return;
            const bool k_whole = valid == kPage && !holds_nan(k);
            if (kPart == 4) {
                if (k_whole) scores<true>(k, 0, valid, s);
                else scores<false>(k, 0, valid, s);
                release();
                if (t_issue < 2 * pages_end) issue(u, policy, once, flag);
                softmax<kPart>(s);
                const uint32_t v = await();
                if (gave_up) return;
                if (valid == kPage && !holds_nan(v)) values<true>(v, 0, valid, s);
                else values<false>(v, 0, valid, s);
                release();
                if (t_issue < 2 * pages_end) issue(u, policy, once, flag);
            } else {
                // both tiles are needed at once
                ++used;
                const uint32_t v = await();
                --used;
                if (gave_up) return;
                const bool whole = k_whole && !holds_nan(v);
                if (whole) {
                    scores<true>(k, 0, valid, s);
                    softmax<kPart>(s);
                    values<true>(v, 0, valid, s);
                    scores<true>(k, kPart, valid, s);
                    softmax<kPart>(s);
                    values<true>(v, kPart, valid, s);
                } else {
#pragma unroll 1
                    for (int j0 = 0; 16 * j0 < valid; j0 += kPart) {
                        scores<false>(k, j0, valid, s);
                        softmax<kPart>(s);
                        values<false>(v, j0, valid, s);
                    }
                }
                used += 2;
                __syncwarp();
                if (t_issue < 2 * pages_end) issue(u, policy, once, flag);
                if (t_issue < 2 * pages_end) issue(u, policy, once, flag);
            }
        }
    }

    // ---- the tree's own keys and values (bf16), nodes n0 .. n1 - 1, 16 at a time.  `parents`, `masks`: this warp's own.
    __device__ __forceinline__ void tree(const Unit &u, int n0, int n1, unsigned char *parents, uint64_t *masks, int &flag) {
        const int32_t *par = p.parent + (size_t)u.b * p.T;
        bool bad = false;
        for (int j = lane; j < p.T; j += 32) {
            const int a = par[j];
            bad |= !(j == 0 ? a == -1 : a >= 0 && a < j);
            parents[j] = (unsigned char)a;   // -1: 255
        }
        __syncwarp();
        if (__any_sync(0xffffffffu, bad)) {
            flag |= kBadTree;
            return;
        }
        if (lane < S::kRows) {   // the nodes that each row sees
            const int r = u.rt * S::kRows + lane;
            uint64_t lo = 0, hi = 0;
            if (r < p.T * p.G) {
                const int j = node_of(p, r);
                if (p.anc) {
                    lo = p.anc[((size_t)u.b * p.T + j) * 2];
                    hi = p.anc[((size_t)u.b * p.T + j) * 2 + 1];
                } else {
                    for (int i = j; i != 255; i = parents[i]) {   // (strictly falling on a valid tree)
                        if (i < 64) lo |= 1ull << i;
                        else hi |= 1ull << (i - 64);
                    }
                }
            }
            masks[2 * lane] = lo;
            masks[2 * lane + 1] = hi;
        }
        __syncwarp();
#pragma unroll 1
        for (int n = n0; n < n1; n += 16) {
            const int left = n1 - n;
            float s[1][NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[0][nt][i] = 0.f;
            const __nv_bfloat16 *k = p.k_tree + (((size_t)u.b * p.T + n) * p.Hkv + u.h) * D + c * (D / 4);
            const uint4 *ka = reinterpret_cast<const uint4 *>(k + (size_t)g * p.Hkv * D), *kb = reinterpret_cast<const uint4 *>(k + (size_t)(g + 8) * p.Hkv * D);
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                const uint4 a = g < left ? ka[x] : make_uint4(0, 0, 0, 0), b = g + 8 < left ? kb[x] : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma(s[0][nt], a.x, b.x, a.y, b.y, qf[2 * x][nt][0], qf[2 * x][nt][1]);
                    mma(s[0][nt], a.z, b.z, a.w, b.w, qf[2 * x + 1][nt][0], qf[2 * x + 1][nt][1]);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t sees = (uint32_t)(masks[2 * (8 * nt + 2 * c + e) + (n >> 6)] >> (n & 63));
                    if (g >= left || !((sees >> g) & 1u)) s[0][nt][e] = -INFINITY;
                    if (g + 8 >= left || !((sees >> (g + 8)) & 1u)) s[0][nt][2 + e] = -INFINITY;
                }
            softmax<1>(s);
            uint32_t b[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                b[nt][0] = transposed(pack(s[0][nt][0], s[0][nt][1]));
                b[nt][1] = transposed(pack(s[0][nt][2], s[0][nt][3]));
            }
            const __nv_bfloat16 *v = p.v_tree + (((size_t)u.b * p.T + n) * p.Hkv + u.h) * D + g * kOwn;
            bool dirty = false;
#pragma unroll
            for (int x = 0; x < kOwn / 8; ++x) {   // eight elements of two pairs of nodes at a time
                uint4 w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = 2 * c + (i & 1) + 8 * (i >> 1);
                    w[i] = make_uint4(0, 0, 0, 0);
                    if (key < left) w[i] = *reinterpret_cast<const uint4 *>(v + (size_t)key * p.Hkv * D + 8 * x);
                    dirty |= clean(w[i]);
                }
                const uint32_t a[4][4] = {{w[0].x, w[0].y, w[0].z, w[0].w}, {w[1].x, w[1].y, w[1].z, w[1].w}, {w[2].x, w[2].y, w[2].z, w[2].w}, {w[3].x, w[3].y, w[3].z, w[3].w}};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma(o[4 * x + i][nt], __byte_perm(a[0][i], a[1][i], 0x5410), __byte_perm(a[0][i], a[1][i], 0x7632), __byte_perm(a[2][i], a[3][i], 0x5410),
                            __byte_perm(a[2][i], a[3][i], 0x7632), b[nt][0], b[nt][1]);
            }
            // Infinities and NaN among the values: 0 times them is NaN, so they were left out of the product; the rows that see them get them.
            if (__any_sync(0xffffffffu, dirty)) {
#pragma unroll 1
                for (int k = 0; k < min(left, 16); ++k) {
                    const uint32_t *row = reinterpret_cast<const uint32_t *>(v + (size_t)k * p.Hkv * D);
#pragma unroll
                    for (int x = 0; x < kOwn / 2; ++x) {
                        const uint32_t w = row[x];
                        const float lo = nonfinite(w << 16) ? bf16lo(w) : 0.f, hi = nonfinite(w) ? bf16hi(w) : 0.f;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const bool sees = (masks[2 * (8 * nt + 2 * c + e) + (n >> 6)] >> ((n & 63) + k)) & 1;
                                if (sees) {
                                    o[x][nt][e] += lo;
                                    o[x][nt][2 + e] += hi;
                                }
                            }
                    }
                }
            }
        }
    }

    // ---- results.  Lane (g, c) has of rows 2 c and 2 c + 1 of each 8 the elements g D/8 .. + D/8 - 1: 2 x and 2 x + 1 in tile x.
    __device__ __forceinline__ void sum_up() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 4);
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 8);
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 16);
            }
    }
    __device__ __forceinline__ void write_rows(const Unit &u, int flag) {
        note(p, u.b, flag, lane);
        const int live = live_rows<NT>(p, u.rt);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * nt + 2 * c + e;
                if (r >= live) continue;
                const size_t row = out_row<NT>(p, u.b, u.h, u.rt, r);
                const float inv = flag || l[nt][e] == 0.f ? 0.f : 1.f / l[nt][e];   // (a row that sees nothing: zeros)
                uint4 *dst = reinterpret_cast<uint4 *>(p.out + row * D + g * kOwn);
#pragma unroll
                for (int x = 0; x < kOwn / 8; ++x) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = flag ? 0u : pack(o[4 * x + i][nt][e] * inv, o[4 * x + i][nt][2 + e] * inv);
                    dst[x] = make_uint4(w[0], w[1], w[2], w[3]);
                }
                if (p.lse && g == 0) p.lse[row] = flag ? 0.f : fmaf(m[nt][e], p.scale, log2f(l[nt][e]) * 0.6931471805599453f);
            }
    }
    // The worker's share of a unit: O to dst [rows][D], (m, l) to ml [rows].
    __device__ __forceinline__ void write_share(const Unit &u, float *dst, float2 *ml) {
        const int live = live_rows<NT>(p, u.rt);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * nt + 2 * c + e;
                if (r >= live) continue;
                float4 *at = reinterpret_cast<float4 *>(dst + (size_t)r * D + g * kOwn);
#pragma unroll
                for (int x = 0; x < kOwn / 4; ++x) at[x] = make_float4(o[2 * x][nt][e], o[2 * x][nt][2 + e], o[2 * x + 1][nt][e], o[2 * x + 1][nt][2 + e]);
                if (g == 0) ml[r] = make_float2(m[nt][e], l[nt][e]);
            }
    }
    // What becomes of a unit when its tiles in this range are done: it is whole, or there is a share and, from the worker that begins it, a task.
    __device__ __forceinline__ void finish(const Unit &u, const List &list, int worker, ShareTask *task, int flag) {
        sum_up();
        if (u.t0 == 0 && u.t1 == u.ntiles) {
            write_rows(u, flag);
            return;
        }
        const int share = 2 * worker + (u.t0 == 0 ? 1 : 0);
        write_share(u, p.partial_o + (size_t)share * S::kRows * D, p.partial_ml + (size_t)share * S::kRows);
        if (lane == 0) p.flags[share] = flag;
        if (u.t0 != 0) return;
        const int last = list.worker_of(u.last_entry(kUnitCost));
        if (lane == 0) *task = ShareTask{u.b, u.h, u.rt, live_rows<NT>(p, u.rt), worker, last};
    }
    // The block does not end under its own copies.
    __device__ __forceinline__ void drain() {
        if (!gave_up) return;
        const uint64_t t0 = globaltimer_ns();
        for (; used < issued; ++used)
            while (!mbar_try_wait(bars + (used % S::kSlots) * 8, (used / S::kSlots) & 1) && globaltimer_ns() - t0 < 20000000ull) {
            }
    }
};

template <int D, int NT>
__global__ void __launch_bounds__(Shape<NT>::kThreads, 1) q4_attn_list_kernel(const __grid_constant__ Q4AttnParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    using S = Shape<NT>;
    using C = Cfg<D, NT>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Worker<D, NT> k(p);
    k.init(smem, warp);
    pdl_wait();
    pdl_launch_dependents();

    __shared__ int warp_sum[S::kWarps];
    List list;
    list.cost = kUnitCost;
    list.pages = list.weight = 1;
    list.n_wide = p.n_rt;
    list.narrow = 0;
    list.tree_tiles = (p.T + kPage - 1) / kPage;
    Seqs seqs;
    make_list<S::kWarps>(p, list, seqs, reinterpret_cast<int2 *>(smem + C::kOffPrefix), warp_sum);
    // fewer workers when there is little to do, spread over the thread blocks
    list.per_block = max(1, min(S::kWarps, list.W / (kMinEntries * p.n_ctas)));
    list.cut(list.per_block * max(1, min(p.n_ctas, list.W / (kMinEntries * list.per_block))));
    reject_lengths<D>(p, blockIdx.x * S::kWarps + warp, p.n_ctas * S::kWarps, lane);

    ShareTask *task = p.tasks + blockIdx.x * S::kWarps + warp;
    if (lane == 0) task->first = -1;
    __syncthreads();
    const int worker = blockIdx.x * list.per_block + warp;
    if (warp < list.per_block && worker < list.n_workers && list.W > 0) {
        int w = list.begin(worker);
        const int w_end = list.begin(worker + 1);
        const uint64_t policy = l2_policy_evict_first();
        const bool once = p.n_rt == 1;   // no other unit reads these pages
        unsigned char *parents = smem + C::kOffParents + warp * kMaxNodes;
        uint64_t *masks = reinterpret_cast<uint64_t *>(smem + C::kOffMasks) + warp * S::kRows * 2;
        Unit u;
        u.any = false;
        int flag = 0, pages_end = 0;
        for (;;) {
            // The next unit's first tiles are on their way before this one's results are written.
            Unit coming;
            int coming_flag = 0, coming_end = 0;
            coming.any = false;
            while (w < w_end && !coming.any) {
                coming = unit_at(p, list, seqs, w, w_end, lane);
                w += coming.entries;
            }
            if (coming.any && !k.gave_up) {
                coming_end = min(coming.npages, coming.t1);
                if (p.num_pages == 0 && coming.t0 < coming_end) {   // no pool to read from
                    coming_flag |= kBadPage;
                    coming_end = coming.t0;
                }
                k.start(coming, coming_end, policy, once, coming_flag);
            }
            if (u.any) {
                k.finish(u, list, worker, task, flag);
            }
            if (!coming.any) break;
            u = coming;
            flag = coming_flag;
            pages_end = coming_end;
            k.begin(u);
            // (the tree first: its rows come while the first tiles are on their way)
            const int n0 = max(0, u.t0 - u.npages) * kPage, n1 = min(p.T, (u.t1 - u.npages) * kPage);
            if (n1 > n0) k.tree(u, n0, n1, parents, masks, flag);
            if (!k.gave_up) k.walk(u, pages_end, policy, once, flag);
            flag = __reduce_or_sync(0xffffffffu, flag);
            if (k.gave_up || worker == p.give_up) flag |= kGaveUp;   // (the rest of the range is given up with the unit)
        }
        k.drain();
    }
}

// Units that several workers have shares of: those that the workers of block blockIdx.x of the attention begin, some rows of each, a thread to four
// elements of a row.  Four groups of threads take a unit each; a long one (at most one of a block's workers begins a unit that goes on behind
// the block) is all groups' at once.  (Single tokens, 32/8/128, by all groups and by one: one on 32768, 300 shares a unit, 28.4 and 44.9 us; 16 on 4096, 18 shares, 27.5
// and 28.7.  Fewer than 17 may be several in a block.)
constexpr int kGroup = 128, kGroups = 4, kLongTask = 16;
template <int D, int NT>
__global__ void __launch_bounds__(kGroup *kGroups) q4_attn_list_merge_kernel(const __grid_constant__ Q4AttnParams p) {
    using S = Shape<NT>;
    constexpr int kRows = S::kRows;
    const int tid = threadIdx.x, group = tid / kGroup, r = blockIdx.y * (4 * kGroup / D) + tid % kGroup / (D / 4), c = tid % (D / 4);
    __shared__ Part parts[kGroup * kGroups];
    pdl_wait();
    pdl_launch_dependents();
    const ShareTask *tasks = p.tasks + blockIdx.x * S::kWarps;
    auto merge = [&](const ShareTask &t, int n0, int n1) {
        return merge_shares(p, t, n0, n1, kRows, r, [&](int share) { return reinterpret_cast<const float4 *>(p.partial_o)[((size_t)share * kRows + r) * (D / 4) + c]; });
    };
    const int lane = tid & 31, own_first = lane < S::kWarps ? tasks[lane].first : -1, own_last = lane < S::kWarps ? tasks[lane].last : -1;
    const bool is_long = own_first >= 0 && own_last - own_first >= kLongTask;
    const unsigned long_ones = __ballot_sync(0xffffffffu, is_long);
    unsigned others = __ballot_sync(0xffffffffu, own_first >= 0 && !is_long);
#pragma unroll 1
    for (int n = 0; others; ++n, others &= others - 1) {
        if (n % kGroups != group) continue;
        const ShareTask t = tasks[__ffs(others) - 1];
        if (r < t.rows) put_merged<D>(p, t, kRows, r, c, merge(t, 0, t.last - t.first + 1));
    }
    if (!long_ones) return;
    const int long_task = __ffs(long_ones) - 1;
    const ShareTask t = tasks[long_task];
    const int count = t.last - t.first + 1, each = (count + kGroups - 1) / kGroups;
    if (r < t.rows) parts[tid] = merge(t, group * each, min(count, (group + 1) * each));
    __syncthreads();
    if (group != 0 || r >= t.rows) return;
    Part y = parts[tid];
#pragma unroll
    for (int i = 1; i < kGroups; ++i) y.add(parts[tid + i * kGroup], p.scale_log2);
    put_merged<D>(p, t, kRows, r, c, y);
}

// The other form: a cluster of thread blocks per sequence, p.split of them for each of its units.
template <int D, int NT>
__global__ void __launch_bounds__(Shape<NT>::kThreads, 1) q4_attn_alone_kernel(const __grid_constant__ Q4AttnParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    using S = Shape<NT>;
    using C = Cfg<D, NT>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Worker<D, NT> k(p);
    k.init(smem, warp);
    __shared__ int flags;
    if (tid == 0) flags = 0;
    __syncthreads();   // before any warp raises one
    pdl_wait();
    pdl_launch_dependents();
    const int size = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
    const int n_rt = p.n_rt, unit = rank / p.split, piece = rank - unit * p.split;
    Unit u;
    u.b = blockIdx.x / size;
    u.h = unit / n_rt;
    u.rt = unit - u.h * n_rt;
    u.L = p.seq_lens[u.b];
    const bool ok = length_ok(p, u.L);
    u.npages = ok ? (u.L + kPage - 1) / kPage : 0;
    u.ntiles = ok ? u.npages + (p.T + kPage - 1) / kPage : 0;
    const int workers = p.split * S::kWarps, mine = piece * S::kWarps + warp;
    u.t0 = mul_div(mine, u.ntiles, workers);
    u.t1 = mul_div(mine + 1, u.ntiles, workers);
    u.any = u.t1 > u.t0;
    int flag = 0;
    float *share = reinterpret_cast<float *>(smem + warp * C::kRingBytes);   // the ring, when no copy is under way any more
    float2 *ml_all = reinterpret_cast<float2 *>(smem + C::kOffShares), *ml_mine = ml_all + warp * S::kRows;
    if (u.any) {
        const uint64_t policy = l2_policy_evict_first();
        const bool once = n_rt == 1;
        int pages_end = min(u.npages, u.t1);
        if (p.num_pages == 0 && u.t0 < pages_end) {   // no pool to read from
            flag |= kBadPage;
            pages_end = u.t0;
        }
        k.start(u, pages_end, policy, once, flag);
        k.begin(u);
        const int n0 = max(0, u.t0 - u.npages) * kPage, n1 = min(p.T, (u.t1 - u.npages) * kPage);
        if (n1 > n0)
            k.tree(u, n0, n1, smem + C::kOffParents + warp * kMaxNodes, reinterpret_cast<uint64_t *>(smem + C::kOffMasks) + warp * S::kRows * 2, flag);
        k.walk(u, pages_end, policy, once, flag);
        flag = __reduce_or_sync(0xffffffffu, flag);
        if (k.gave_up || (int)blockIdx.x * S::kWarps + warp == p.give_up) flag |= kGaveUp;
        k.drain();
        k.sum_up();
        k.write_share(u, share, ml_mine);
    } else {
        for (int i = lane; i < S::kRows * D / 4; i += 32) reinterpret_cast<float4 *>(share)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (lane < S::kRows) ml_mine[lane] = make_float2(-INFINITY, 0.f);
        // (without a tile nobody looks at the tree: the first worker does)
        if (!ok && mine == 0) flag = tree_ok(p, u.b, lane) ? kBadLength : kBadTree;
    }
    if (flag && lane == 0) atomicOr(&flags, flag);
    __syncthreads();
    const int live = live_rows<NT>(p, u.rt), block_flag = ok ? flags : flags | kBadLength;
    // the block's shares, a row to a warp
    for (int r = warp; r < live; r += S::kWarps) {
        const Row x = merge_row<D>(
            S::kWarps, p.scale_log2, [&](int w) { return ml_all[w * S::kRows + r]; },
            [&](int w) { return *reinterpret_cast<const float4 *>(smem + w * C::kRingBytes + (r * D + lane * 4) * 4); });
        if (p.split == 1) {
            put_row<D>(p, out_row<NT>(p, u.b, u.h, u.rt, r), x, block_flag);
        } else {
            keep_row<D>(p, (size_t)blockIdx.x * S::kRows + r, x);
        }
    }
    if (tid == 0) p.flags[blockIdx.x] = block_flag;
    cluster_arrive_release();
    cluster_wait_acquire();
    const int block0 = blockIdx.x - rank;   // the cluster's first
    if (rank == 0 && warp == 0) {
        const int all = __reduce_or_sync(0xffffffffu, lane < size ? __ldcg(p.flags + block0 + lane) : 0);
        if (lane == 0) p.status[u.b] = code_of_flag(all);
    }
    if (p.split == 1) return;
    // the shares of the unit's blocks, a row to a warp of them
    const int first = block0 + unit * p.split, unit_flag = __reduce_or_sync(0xffffffffu, lane < p.split ? __ldcg(p.flags + first + lane) : 0);
    for (int r = warp * p.split + piece; r < live; r += workers) {
        const Row x = merge_row<D>(
            p.split, p.scale_log2, [&](int w) { return __ldcg(p.partial_ml + (first + w) * S::kRows + r); },
            [&](int w) { return __ldcg(reinterpret_cast<const float4 *>(p.partial_o + ((size_t)(first + w) * S::kRows + r) * D + lane * 4)); });
        put_row<D>(p, out_row<NT>(p, u.b, u.h, u.rt, r), x, unit_flag);
    }
}

__global__ void __launch_bounds__(1024) q4_attn_status_kernel(int32_t *status, int B) {
    pdl_launch_dependents();   // the attention may be set up meanwhile; it waits for this kernel's end
    pdl_wait();
    for (int b = threadIdx.x; b < B; b += 1024) status[b] = READER_OK;
}

// Thread blocks of a unit in the alone form, 0 if the call is not one for it: the units of a sequence have to fit a cluster, the clusters the GPU all at once (8
// single tokens on 2048, 32/8/128: eight clusters of 16 blocks in two turns 20.8 us, of 8 in one 13.9; 4 of them 11.2 and 13.5), and,
// going by the page table's width, a worker gets at most `most` tiles.  Few rows: six.  The width is what a sequence may grow to, and short ones gain: 511 positions
// (32/8/128) behind a table of any allowed width take 7.2 to 9.0 us instead of the list form's 12.8, of eight sequences 8.3 instead of 18.0.  Those that fill their table gain
// up to two tiles a worker (4032 positions 14.2 instead of 15.6, eight of 1984 13.3 instead of 16.8; one KV head's 98240, six tiles, 31.9 instead of 33.2), eight
// up to four (4032 positions 21.9 instead of 22.9), and lose at six (12224 positions 30.8 instead of 17.6, eight of 6080 30.3 instead of 27.2); at seven the alone form
// would lose by as much or more (34.9 instead of 17.6, 34.5 instead of 27.7).
constexpr int kAloneTiles = 6, kAloneTilesManyRows = 2;
template <int NT>
int alone_split(const Q4AttnParams &p, const Q4RowsKernels &k, int most) {
    using S = Shape<NT>;
    const int64_t units = (int64_t)p.Hkv * ((p.T * p.G + S::kRows - 1) / S::kRows), tiles = p.max_pages + (p.T + kPage - 1) / kPage;
    auto fits = [&](int64_t blocks) { return blocks <= kQ4MaxCluster && p.B <= k.clusters[blocks]; };
    if (!fits(units)) return 0;
    int split = 1;
    while (fits(2 * split * units) && tiles > split * S::kWarps) split *= 2;
    return tiles <= (int64_t)most * split * S::kWarps ? split : 0;
}

template <int D, int NT>
reader_status set_up(Q4RowsKernels *k) {
    using S = Shape<NT>;
    using C = Cfg<D, NT>;
    if (!k->set) {
        if (cudaFuncSetAttribute(q4_attn_list_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess ||
            cudaFuncSetAttribute(q4_attn_alone_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) != cudaSuccess ||
            cudaFuncSetAttribute(q4_attn_alone_kernel<D, NT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
            cudaGetLastError();
            return READER_ERR_CUDA;
        }
        for (int blocks = 1; blocks <= kQ4MaxCluster; ++blocks) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)blocks);
            cfg.blockDim = dim3(S::kThreads);
            cfg.dynamicSmemBytes = C::kSmem;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = (unsigned)blocks;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, q4_attn_alone_kernel<D, NT>, &cfg) != cudaSuccess) {
                cudaGetLastError();
                return READER_ERR_CUDA;
            }
            k->clusters[blocks] = (int16_t)n;
        }
        k->set = true;
    }
    return READER_OK;
}

template <int D, int NT>
reader_status launch(Q4RowsKernels *k, Q4AttnParams p, int n_sm, cudaStream_t st) {
    using S = Shape<NT>;
    using C = Cfg<D, NT>;
    if (reader_status e = set_up<D, NT>(k)) return e;
    p.n_rt = (p.T * p.G + S::kRows - 1) / S::kRows;
    p.split = alone_split<NT>(p, *k, kAloneTiles);
    if (p.split) {
        const int blocks = p.Hkv * p.n_rt * p.split;   // of a sequence
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(p.B * blocks));
        cfg.blockDim = dim3(S::kThreads);
        cfg.dynamicSmemBytes = C::kSmem;
        cfg.stream = st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)blocks;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        if (cudaLaunchKernelEx(&cfg, q4_attn_alone_kernel<D, NT>, p) != cudaSuccess) {
            cudaGetLastError();
            return READER_ERR_CUDA;
        }
        return READER_OK;
    }
    p.n_ctas = n_sm;
    launch_q4_attn_status(p, st);
    launch_pdl(q4_attn_list_kernel<D, NT>, dim3((unsigned)n_sm), dim3(S::kThreads), (size_t)C::kSmem, st, p);
    static_assert(S::kWarps <= kLongTask && S::kWarps <= kQ4Ranges && 2 * S::kWarps * S::kRows <= kQ4ShareRows, "workspace");
    launch_pdl(q4_attn_list_merge_kernel<D, NT>, dim3((unsigned)n_sm, (unsigned)((std::min(S::kRows, p.T * p.G) * D + 4 * kGroup - 1) / (4 * kGroup))), dim3(kGroup * kGroups), 0,
               st, p);
    return READER_OK;
}

}  // namespace

void launch_q4_attn_status(const Q4AttnParams &p, cudaStream_t st) { launch_pdl(q4_attn_status_kernel, dim3(1), dim3(1024), 0, st, p.status, p.B); }

reader_status q4_attn_rows_faster(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, bool *yes) {
    *yes = p.T * p.G <= kQ4FewRows;
    if (*yes) return READER_OK;
    // With many rows the form of one launch saves two, and its workers need longer for a tile: for calls that leave two thirds of the GPU idle either way.
    const int64_t units = (int64_t)p.B * p.Hkv * ((p.T * p.G + 15) / 16);
    if (3 * units > n_sm) return READER_OK;
    Q4RowsKernels *k = &attr->rows[p.D == 128 ? 3 : 1];
    if (reader_status e = p.D == 128 ? set_up<128, 2>(k) : set_up<64, 2>(k)) return e;
    *yes = alone_split<2>(p, *k, kAloneTilesManyRows) != 0;
    return READER_OK;
}

reader_status launch_q4_attn_rows(Q4AttrSet *attr, const Q4AttnParams &p, int n_sm, cudaStream_t st) {
    const bool few = p.T * p.G <= 8;
    if (p.D == 128) return few ? launch<128, 1>(&attr->rows[2], p, n_sm, st) : launch<128, 2>(&attr->rows[3], p, n_sm, st);
    return few ? launch<64, 1>(&attr->rows[0], p, n_sm, st) : launch<64, 2>(&attr->rows[1], p, n_sm, st);
}

}  // namespace reader

// Tree-masked attention over a 4-bit cache for few query rows (reader_q4_verify_attn): single tokens, small trees.
//
// A unit is (sequence, KV head, 16 query rows).  Bound: bytes, 72 D of every 64 positions and head, if the numbers become
// operands fast enough.  So they never leave a warp: each warp is a worker of its own that brings tiles (one page of keys and
// values of one head, 72 D bytes) into its own ring in shared memory by bulk copies and computes S = Q K^T and O += P V with
// m16n8k16 products whose B fragments it unpacks in registers, two bf16 in 2.75 instructions; the pages are laid out so that
// a lane's words, and their scales, are one or two 16-byte loads.  (Feeding tcgen05.mma instead means writing every tile in
// bf16 to shared memory and reading it back: worth it once many rows share it, not for 4 or 16.)  A fragment's column order is
// free as long as both operands agree: of the elements, lane (g, c) = (lane / 4, lane % 4) has D/4 consecutive ones of a key,
// and D/8 consecutive ones of a pair of values, with one or two scales; P comes out of the score product in the place where the
// value product wants it.
//
// Work.  The units, each preceded by kUnitCost entries for its start and end, form one flat list of tiles that is cut into equal
// ranges, one per worker.  Every thread block makes the list's prefix sums from seq_lens itself.  A unit that lies in several
// ranges leaves shares (m, l, O) in the workspace; the last to arrive of a group of 16 merges the group, the last group the
// unit, always in the order of the shares, whoever comes last.  The counters are zeroed by a launch in front.
//
// What is checked where: lengths by every block, page ids by the worker that reads them, a tree by the worker of the unit's
// tree tiles; what is wrong travels with the share and zeroes the unit's rows.  Bytes behind a sequence's end never reach a
// product: their scores are replaced by -inf and their values' scale by 0.  Every wait is bounded; a worker that gives up says so
// in its share, waits (bounded) for its copies and goes on without them.
#include <climits>

#include "ptx_sm100.cuh"
#include "q4_attn.cuh"
#include "q4_format.cuh"

namespace reader {
namespace {

using namespace ptx;

constexpr int kThreads = kQ4Warps * 32;
constexpr int kStages = 2;
constexpr int kUnitCost = 2;       // entries that stand for a unit's start and end
constexpr int kMinEntries = 4;     // a smaller range costs more in merging than it saves in time
constexpr int kOneLevel = 16;      // up to so many shares are merged at once, more in groups
constexpr int kMaxShares = 32 * 32;
constexpr int kPrefix = 1024;      // entries of the prefix table in shared memory
constexpr float kRaiseBy = 8.f;    // log2 units by which a score may exceed the maximum in use
constexpr uint64_t kWaitLimitNs = 1000000000ull;
constexpr int kBadTree = 1, kBadPage = 2, kGaveUp = 4;

template <int D>
struct Cfg {
    static constexpr int kTile = q4::tile_bytes(D);
    static constexpr int kStageBytes = 2 * kTile;
    static constexpr int kRing = kQ4Warps * kStages * kStageBytes;
    static constexpr int kOffBars = kRing;
    static constexpr int kOffParents = kOffBars + kQ4Warps * kStages * 8;
    static constexpr int kOffPrefix = kOffParents + kQ4Warps * kMaxNodes;
    static constexpr int kSmem = kOffPrefix + (kPrefix + 1) * 4;
    static_assert(kSmem <= 227 * 1024, "shared memory");
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy, bool streamed) {
    if (streamed)
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
                     "l"(src), "r"(bytes), "r"(bar), "l"(policy)
                     : "memory");
    else
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(a));
    return x;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t x;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(a));
    return x;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 x;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(a));
    return x;
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// A pair of scales as bf16 and the pair times -24.
struct Scale2 {
    uint32_t s, m24;
};
constexpr uint32_t kScaleOne = (uint32_t)((127 - q4::kScaleBias) << 7) * 0x10001u;
// codes: two of them, in bits 0-7 and 16-23
__device__ __forceinline__ Scale2 scale2(uint32_t codes, bool any_nan) {
    Scale2 r;
    r.s = codes * 16u + kScaleOne;
    if (any_nan) {
        if ((codes & 0xffffu) == q4::kNanCode) r.s |= 0x7fffu;
        if ((codes >> 16) == q4::kNanCode) r.s |= 0x7fff0000u;
    }
    r.m24 = mul_bf16x2(r.s, 0xc1c0c1c0u);
    return r;
}
// Whether one of eight codes is kNanCode (four bytes 255 have all bits set in some byte).
__device__ __forceinline__ bool has_nan(uint32_t a, uint32_t b) { return (__vcmpeq4(a, 0xffffffffu) | __vcmpeq4(b, 0xffffffffu)) != 0; }
// Pair i of a word: numbers n in the mantissas of 16 + n, times the scales, minus 24 of them: (n - 8) s, exactly.
template <int i>
__device__ __forceinline__ uint32_t pair(uint32_t w, const Scale2 &s) {
    const uint32_t x = i ? __funnelshift_r(w, w, 4 * i) : w;
    return fma_bf16x2((x & 0x00780078u) | 0x41804180u, s.s, s.m24);
}

// ---- the work list
struct Unit {
    int b, h, rt, L, npages, ntiles;
    int t0, t1;              // this range's tiles
    int w0;                  // flat index of the unit's first entry
    int entries;             // of the flat list that this range has of the unit
    bool any;
};

struct List {
    int W, n_workers, per_seq, tree_tiles, step;   // step: sequences per entry of the prefix table
    __device__ __forceinline__ int begin(int worker) const { return mul_div(worker, W, n_workers); }
    // the worker whose range holds entry w
    __device__ __forceinline__ int worker_of(int w) const {
        int c = (int)((float)w * (float)n_workers / (float)W);
        c = max(0, min(c, n_workers - 1));
        while (c + 1 < n_workers && begin(c + 1) <= w) ++c;
        while (c > 0 && begin(c) > w) --c;
        return c;
    }
};

__device__ __forceinline__ bool length_ok(const Q4AttnParams &p, int L) { return L >= 0 && (int64_t)L <= (int64_t)p.max_pages * kPage; }
__device__ __forceinline__ int entries_of(const Q4AttnParams &p, const List &l, int L) {
    return length_ok(p, L) ? ((L + kPage - 1) / kPage + l.tree_tiles + kUnitCost) * l.per_seq : 0;
}

// The part of the list from w on that lies in one unit (and before w_end).  Warp-collective.
__device__ __forceinline__ Unit unit_at(const Q4AttnParams &p, const List &l, const int32_t *prefix, int w, int w_end, int lane) {
    Unit u;
    // the last prefix entry that is not behind w
    const int n = (p.B + l.step - 1) / l.step;
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= w) lo = mid; else hi = mid;
    }
    int start = prefix[lo], b = lo * l.step;
    if (l.step == 1) {
        u.L = p.seq_lens[b];
    } else {   // at most 64 sequences from there on
        int left = min(l.step, p.B - b);
        for (;;) {
            const int L = lane < left ? p.seq_lens[b + lane] : -1;
            const int e = lane < left ? entries_of(p, l, L) : 0;
            int incl = e;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int t = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += t;
            }
            const unsigned here = __ballot_sync(0xffffffffu, e > 0 && start + incl > w);
            if (here) {
                const int j = __ffs(here) - 1;
                start += __shfl_sync(0xffffffffu, incl - e, j);
                u.L = __shfl_sync(0xffffffffu, L, j);
                b += j;
                break;
            }
            start += __shfl_sync(0xffffffffu, incl, 31);
            b += 32;
            left -= 32;
            if (left <= 0) break;   // (cannot be: w lies before the next entry)
        }
    }
    u.b = b;
    u.npages = (u.L + kPage - 1) / kPage;
    u.ntiles = u.npages + l.tree_tiles;
    const int per_unit = u.ntiles + kUnitCost, local = w - start, unit = local / per_unit, pos = local - unit * per_unit;
    const int n_rt = l.per_seq / p.Hkv;
    u.h = unit / n_rt;
    u.rt = unit - u.h * n_rt;
    const int pos_end = min(per_unit, pos + (w_end - w));
    u.entries = pos_end - pos;
    u.w0 = w - pos;
    u.t0 = max(0, pos - kUnitCost);
    u.t1 = max(0, pos_end - kUnitCost);
    u.any = u.t1 > u.t0;
    return u;
}

// ---- rows of a unit
__device__ __forceinline__ size_t out_row(const Q4AttnParams &p, int b, int h, int rt, int r) {
    const int row = rt * kQ4Rows + r, j = row / p.G;
    return ((size_t)b * p.T + j) * p.Hq + h * p.G + (row - j * p.G);
}
__device__ __forceinline__ int live_rows(const Q4AttnParams &p, int rt) { return min(kQ4Rows, p.T * p.G - rt * kQ4Rows); }
__device__ __forceinline__ void note(const Q4AttnParams &p, int b, int flag, int lane) {
    if (flag && lane == 0) atomicMax(p.status + b, (flag & kBadTree) ? READER_ERR_BAD_TREE : (flag & kBadPage) ? READER_ERR_BAD_PAGE : READER_ERR_TIMEOUT);
}

    // (Not inlined: its registers are not those of a worker's loop.)  Merges the shares in slots first, then base + 2 k for k = 1 .. count - 1 (times `apart`), into the result or into slot `first`.
    // (count <= 32.)  A share whose maximum is -inf has weight 0 and is still added, so that a NaN in it stays.
    template <int D>
__device__ __noinline__ void merge(const Q4AttnParams &p, int b, int h, int rt, int first, int base, int apart, int count, bool final) {
    const int lane = threadIdx.x & 31;
        auto slot_of = [&](int k) { return k == 0 ? first : base + 2 * apart * k; };
        int flag = lane < count ? __ldcg(p.flags + slot_of(lane)) : 0;
        flag = __reduce_or_sync(0xffffffffu, flag);
        const int live = live_rows(p, rt);
        if (final) note(p, b, flag, lane);
        constexpr int kRows = 4;       // rows under way at once
        const bool has = lane * 4 < D;
#pragma unroll 1
        for (int r0 = 0; r0 < live; r0 += kRows) {
            float weight[kRows], total[kRows], top[kRows];
            float4 acc[kRows];
            float2 ml[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                ml[i] = make_float2(-INFINITY, 0.f);
                if (lane < count && r0 + i < live) ml[i] = __ldcg(p.partial_ml + slot_of(lane) * kQ4Rows + r0 + i);
                acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                float t = ml[i].x;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
                top[i] = t;
                weight[i] = ml[i].x == -INFINITY ? 0.f : ml[i].x == t ? 1.f : ex2((ml[i].x - t) * p.scale_log2);
                t = ml[i].y * weight[i];
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
                total[i] = t;
            }
#pragma unroll 1
            for (int k0 = 0; k0 < count; k0 += 4) {
                float4 x[4][kRows];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        x[k][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (has && k0 + k < count && r0 + i < live)
                            x[k][i] = __ldcg(reinterpret_cast<const float4 *>(p.partial_o + ((size_t)slot_of(k0 + k) * kQ4Rows + r0 + i) * D + lane * 4));
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        const float w = __shfl_sync(0xffffffffu, weight[i], min(k0 + k, 31));   // (behind the last share: 0 times 0)
                        acc[i].x = fmaf(x[k][i].x, w, acc[i].x);
                        acc[i].y = fmaf(x[k][i].y, w, acc[i].y);
                        acc[i].z = fmaf(x[k][i].z, w, acc[i].z);
                        acc[i].w = fmaf(x[k][i].w, w, acc[i].w);
                    }
            }
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int r = r0 + i;
                if (r >= live) continue;
                if (final) {
                    const size_t row = out_row(p, b, h, rt, r);
                    const float inv = total[i] == 0.f ? 0.f : 1.f / total[i];
                    if (has)
                        *reinterpret_cast<uint2 *>(p.out + row * D + lane * 4) =
                            flag ? make_uint2(0u, 0u) : make_uint2(pack(acc[i].x * inv, acc[i].y * inv), pack(acc[i].z * inv, acc[i].w * inv));
                    if (p.lse && lane == 0) p.lse[row] = flag ? 0.f : fmaf(top[i], p.scale, log2f(total[i]) * 0.6931471805599453f);
                } else {
                    if (has) *reinterpret_cast<float4 *>(p.partial_o + ((size_t)first * kQ4Rows + r) * D + lane * 4) = acc[i];
                    if (lane == 0) p.partial_ml[first * kQ4Rows + r] = make_float2(top[i], total[i]);
                }
            }
        }
        if (!final) {
            __syncwarp();
            if (lane == 0) p.flags[first] = flag;
        }
    }

// ---- one worker
template <int D>
struct Worker {
    static constexpr int kSteps = D / 16;    // k-steps of the score product; also scale blocks of a head
    static constexpr int kCols = D / 8;      // n-tiles of the value product = value elements of a lane
    const Q4AttnParams &p;
    uint32_t ring, bars;
    int lane, g, c;
    int issued, used;        // tiles, counted over the worker's life
    bool gave_up;
    // the unit's page ids, 32 at a time
    int ids, ids_next, ids_at;

    uint32_t qf[kSteps][4];
    float o[kCols][4];
    float m[2], l[2];        // rows g and g + 8; l: this lane's share

    __device__ __forceinline__ Worker(const Q4AttnParams &p_) : p(p_) {}

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
    __device__ __forceinline__ void start(const Unit &u, int &flag) {
        ids_at = u.t0;
        ids = page_ids(u, u.t0, flag);
        ids_next = page_ids(u, u.t0 + 32, flag);
    }
    __device__ __forceinline__ void issue(const Unit &u, int t, uint64_t policy, bool streamed, int &flag) {
        if (t - ids_at == 32) {
            ids_at = t;
            ids = ids_next;
            ids_next = page_ids(u, t + 32, flag);
        }
        const int page = __shfl_sync(0xffffffffu, ids, t - ids_at);
        if (lane == 0) {
            const int s = issued % kStages;
            const uint32_t bar = bars + s * 8, dst = ring + s * Cfg<D>::kStageBytes;
            const size_t at = ((size_t)page * p.Hkv + u.h) * Cfg<D>::kTile;
            mbar_arrive_expect_tx(bar, Cfg<D>::kStageBytes);
            bulk_load(dst, p.k_pool + at, Cfg<D>::kTile, bar, policy, streamed);
            bulk_load(dst + Cfg<D>::kTile, p.v_pool + at, Cfg<D>::kTile, bar, policy, streamed);
        }
        ++issued;
    }
    __device__ __forceinline__ void await() {
        const uint32_t bar = bars + (used % kStages) * 8, parity = (used / kStages) & 1;
        if (!mbar_try_wait(bar, parity)) {
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar, parity))
                if (globaltimer_ns() - t0 > kWaitLimitNs) {
                    gave_up = true;
                    break;
                }
        }
        gave_up = __any_sync(0xffffffffu, gave_up);
    }

    // ---- queries: lane (g, c) has elements c D/4 .. of rows g and g + 8
    __device__ __forceinline__ void load_queries(const Unit &u) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = u.rt * kQ4Rows + g + 8 * e;
            const bool live = r < p.T * p.G;
            const int j = live ? r / p.G : 0, hq = u.h * p.G + (live ? r - j * p.G : 0);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.q + (((size_t)u.b * p.T + j) * p.Hq + hq) * D + c * (D / 4));
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                const uint4 v = live ? src[x] : make_uint4(0, 0, 0, 0);
                qf[2 * x][e] = v.x; qf[2 * x][2 + e] = v.y;
                qf[2 * x + 1][e] = v.z; qf[2 * x + 1][2 + e] = v.w;
            }
        }
    }

    // ---- softmax of kN n-tiles of scores (columns 8 j + 2 c, + 1): probabilities in place
    template <int kN>
    __device__ __forceinline__ void softmax(float (&s)[kN][4]) {
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            top[0] = max3(top[0], s[j][0], s[j][1]);
            top[1] = max3(top[1], s[j][2], s[j][3]);
        }
        // the maximum in use is raised only when a score exceeds it by 2^8: the vote needs no exchange within the rows
        const float by = kRaiseBy / p.scale_log2;
        if (__any_sync(0xffffffffu, top[0] > m[0] + by || top[1] > m[1] + by)) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
                top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], 2));
                const float now = fmaxf(m[e], top[e]);
                const float f = m[e] == now ? 1.f : ex2((m[e] - now) * p.scale_log2);   // (-inf before the first score: 0)
                m[e] = now;
                l[e] *= f;
#pragma unroll
                for (int n = 0; n < kCols; ++n) {
                    o[n][2 * e] *= f;
                    o[n][2 * e + 1] *= f;
                }
            }
        }
        // The difference to the maximum is taken before the scaling: whatever the scores' size, it is as exact as they are.
        const float2 sc = make_float2(p.scale_log2, p.scale_log2);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        const float from[2] = {m[0] == -INFINITY ? 0.f : -m[0], m[1] == -INFINITY ? 0.f : -m[1]};
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float2 x = __fmul2_rn(__fadd2_rn(make_float2(s[j][2 * e], s[j][2 * e + 1]), make_float2(from[e], from[e])), sc);
                const float2 y = make_float2(ex2(x.x), ex2(x.y));
                s[j][2 * e] = y.x;
                s[j][2 * e + 1] = y.y;
                sum[e] = __fadd2_rn(sum[e], y);
            }
        l[0] += sum[0].x + sum[0].y;
        l[1] += sum[1].x + sum[1].y;
    }

    // ---- one tile of the cache, `valid` of its 64 positions committed: two halves, so that scores take 16 registers
    __device__ __forceinline__ void tile(uint32_t k, int valid) {
        constexpr int kPer = D / 64;   // key scales of a lane and position
        const uint32_t v = k + Cfg<D>::kTile;
        const uint32_t k_row = k + g * (D / 2) + c * (D / 8);
        const uint32_t k_codes = k + q4::scales_at(D) + lane * (8 * kPer);
        // row 4 j + c of D bytes; of its eight chunks the one with this lane's elements
        const uint32_t v_row = v + c * D + q4::v_chunk<D>(c, g) * (D / 8);
        const uint32_t v_codes = v + q4::scales_at(D) + ((D == 128 ? g : g >> 1) * 4 + c) * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (h == 1 && valid <= kPage / 2) break;
            float s[4][4];
            {
                uint32_t cw[2] = {};
                if (D == 128) { const uint2 x = lds64(k_codes + h * 8); cw[0] = x.x; cw[1] = x.y; }
                else cw[0] = lds32(k_codes + h * 4);
                const bool nan = has_nan(cw[0], cw[1]);
#pragma unroll
                for (int jj = 0; jj < 4; ++jj) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[jj][i] = 0.f;
                    uint32_t w[D / 32];
                    load_words(w, k_row + (4 * h + jj) * (8 * D / 2));
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) {
                        // the code of block x / 2 of this position, twice
                        const int byte = jj * kPer + x / 2;
                        const Scale2 sc = scale2(__byte_perm(cw[byte / 4], 0, 0x4040 | (byte % 4) | ((byte % 4) << 8)), nan);
                        mma(s[jj], qf[2 * x], pair<0>(w[x], sc), pair<1>(w[x], sc));
                        mma(s[jj], qf[2 * x + 1], pair<2>(w[x], sc), pair<3>(w[x], sc));
                    }
                }
            }
            if (valid < kPage) {
#pragma unroll
                for (int jj = 0; jj < 4; ++jj) {
                    const int key = 8 * (4 * h + jj) + 2 * c;
                    if (key >= valid) s[jj][0] = s[jj][2] = -INFINITY;
                    if (key + 1 >= valid) s[jj][1] = s[jj][3] = -INFINITY;
                }
            }
            softmax<4>(s);
            {
                const uint2 cx = lds64(v_codes + h * 8);
                const uint32_t cw[2] = {cx.x, cx.y};
                const bool nan = has_nan(cw[0], cw[1]);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t a[4] = {pack(s[2 * t][0], s[2 * t][1]), pack(s[2 * t][2], s[2 * t][3]), pack(s[2 * t + 1][0], s[2 * t + 1][1]),
                                           pack(s[2 * t + 1][2], s[2 * t + 1][3])};
                    uint32_t w[2][D / 32];
                    Scale2 sc[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int jj = 2 * t + e, j = 4 * h + jj;
                        load_words(w[e], v_row + j * (4 * D));
                        sc[e] = scale2(__byte_perm(cw[jj / 2], 0, jj % 2 ? 0x4342 : 0x4140), nan);
                        if (valid < kPage) {   // positions behind the end: scale 0, whatever their code
                            const int key = 8 * j + 2 * c;
                            if (key >= valid) { sc[e].s &= 0xffff0000u; sc[e].m24 &= 0xffff0000u; }
                            if (key + 1 >= valid) { sc[e].s &= 0xffffu; sc[e].m24 &= 0xffffu; }
                        }
                    }
#pragma unroll
                    for (int y = 0; y < D / 32; ++y) {
                        mma(o[4 * y + 0], a, pair<0>(w[0][y], sc[0]), pair<0>(w[1][y], sc[1]));
                        mma(o[4 * y + 1], a, pair<1>(w[0][y], sc[0]), pair<1>(w[1][y], sc[1]));
                        mma(o[4 * y + 2], a, pair<2>(w[0][y], sc[0]), pair<2>(w[1][y], sc[1]));
                        mma(o[4 * y + 3], a, pair<3>(w[0][y], sc[0]), pair<3>(w[1][y], sc[1]));
                    }
                }
            }
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

    // ---- the tree's own keys and values (bf16), nodes n0 .. n1 - 1, 16 at a time.  `parents`: 128 bytes of this warp's own.
    __device__ __forceinline__ void tree(const Unit &u, int n0, int n1, unsigned char *parents, int &flag) {
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
        uint64_t sees[2][2];   // rows g and g + 8: the nodes they see
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = u.rt * kQ4Rows + g + 8 * e;
            sees[e][0] = sees[e][1] = 0;
            if (r >= p.T * p.G) continue;
            const int j = r / p.G;
            if (p.anc) {
                sees[e][0] = p.anc[((size_t)u.b * p.T + j) * 2];
                sees[e][1] = p.anc[((size_t)u.b * p.T + j) * 2 + 1];
            } else {
                for (int i = j; i != 255; i = parents[i]) {   // (strictly falling on a valid tree)
                    if (i < 64) sees[e][0] |= 1ull << i;
                    else sees[e][1] |= 1ull << (i - 64);
                }
            }
        }
#pragma unroll 1
        for (int n = n0; n < n1; n += 16) {
            float s[2][4];
            const int left = n1 - n;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j][i] = 0.f;
                const bool live = 8 * j + g < left;
                const uint4 *src = reinterpret_cast<const uint4 *>(p.k_tree + (((size_t)u.b * p.T + (live ? n + 8 * j + g : n)) * p.Hkv + u.h) * D + c * (D / 4));
#pragma unroll
                for (int x = 0; x < D / 32; ++x) {
                    const uint4 w = live ? src[x] : make_uint4(0, 0, 0, 0);
                    mma(s[j], qf[2 * x], w.x, w.y);
                    mma(s[j], qf[2 * x + 1], w.z, w.w);
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int node = n + 8 * j + 2 * c + (i & 1);
                    const bool seen = 8 * j + 2 * c + (i & 1) < left && ((sees[i >> 1][node >> 6] >> (node & 63)) & 1ull);
                    if (!seen) s[j][i] = -INFINITY;
                }
            softmax<2>(s);
            const uint32_t a[4] = {pack(s[0][0], s[0][1]), pack(s[0][2], s[0][3]), pack(s[1][0], s[1][1]), pack(s[1][2], s[1][3])};
#pragma unroll
            for (int x = 0; x < kCols / 8; ++x) {   // eight elements of two pairs of nodes at a time
                uint4 w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = 2 * c + (i & 1) + 8 * (i >> 1);
                    w[i] = make_uint4(0, 0, 0, 0);
                    if (key < left) w[i] = *reinterpret_cast<const uint4 *>(p.v_tree + (((size_t)u.b * p.T + n + key) * p.Hkv + u.h) * D + g * kCols + 8 * x);
                }
                const uint32_t b[4][4] = {{w[0].x, w[0].y, w[0].z, w[0].w}, {w[1].x, w[1].y, w[1].z, w[1].w}, {w[2].x, w[2].y, w[2].z, w[2].w}, {w[3].x, w[3].y, w[3].z, w[3].w}};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mma(o[8 * x + 2 * i], a, __byte_perm(b[0][i], b[1][i], 0x5410), __byte_perm(b[2][i], b[3][i], 0x5410));
                    mma(o[8 * x + 2 * i + 1], a, __byte_perm(b[0][i], b[1][i], 0x7632), __byte_perm(b[2][i], b[3][i], 0x7632));
                }
            }
        }
    }

    // ---- results.  Lane (g, c) has of rows g and g + 8 the elements c D/4 .. + D/4 - 1: n-tile n, column 2 c + e is element (2 c + e) D/8 + n.
    __device__ __forceinline__ void write_rows(const Unit &u, int flag) {
        note(p, u.b, flag, lane);
        const int live = live_rows(p, u.rt);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = g + 8 * e;
            if (r >= live) continue;
            const size_t row = out_row(p, u.b, u.h, u.rt, r);
            const float inv = flag || l[e] == 0.f ? 0.f : 1.f / l[e];   // (a row that sees nothing: zeros)
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + row * D + c * (D / 4));
#pragma unroll
            for (int x = 0; x < D / 32; ++x) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = 8 * x + 2 * i, n = k % kCols, col = 2 * e + k / kCols;
                    w[i] = flag ? 0u : pack(o[n][col] * inv, o[n + 1][col] * inv);
                }
                dst[x] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (p.lse && c == 0) p.lse[row] = flag ? 0.f : fmaf(m[e], p.scale, log2f(l[e]) * 0.6931471805599453f);
        }
    }
    __device__ __forceinline__ void write_share(const Unit &u, int slot, int flag) {
        const int live = live_rows(p, u.rt);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = g + 8 * e;
            if (r >= live) continue;
            float4 *dst = reinterpret_cast<float4 *>(p.partial_o + ((size_t)slot * kQ4Rows + r) * D + c * (D / 4));
#pragma unroll
            for (int x = 0; x < D / 16; ++x) {
                const int k = 4 * x, n = k % kCols, col = 2 * e + k / kCols;
                dst[x] = make_float4(o[n][col], o[n + 1][col], o[n + 2][col], o[n + 3][col]);
            }
            if (c == 0) p.partial_ml[slot * kQ4Rows + r] = make_float2(m[e], l[e]);
        }
        if (lane == 0) p.flags[slot] = flag;
    }

    // Whether this warp is the last of `count` to arrive; what the others wrote before is visible to it.
    __device__ __forceinline__ bool last_to_arrive(int32_t *counter, int count) {
        __threadfence();
        __syncwarp();
        int before = 0;
        if (lane == 0) before = atomicAdd(counter, 1);
        before = __shfl_sync(0xffffffffu, before, 0);
        if (before != count - 1) return false;
        __threadfence();
        return true;
    }
    __device__ __forceinline__ void finish(const Unit &u, const List &list, int worker, int flag) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
        }
        if (u.t0 == 0 && u.t1 == u.ntiles) {
            write_rows(u, flag);
            return;
        }
        // the unit's shares belong to the workers c0 .. c1; a worker's slots: 2 c + 1 for a unit that it begins, else 2 c
        const int c0 = list.worker_of(u.w0 + kUnitCost), c1 = list.worker_of(u.w0 + kUnitCost + u.ntiles - 1);
        write_share(u, 2 * worker + (u.t0 == 0 ? 1 : 0), flag);
        // up to kOneLevel shares: one group; more: about as many groups as shares in a group
        const int shares = c1 - c0 + 1;
        int size = shares;
        if (shares > kOneLevel) {
            size = 4;
            while (size * size < shares) ++size;
        }
        const int groups = (shares + size - 1) / size, group = (worker - c0) / size, lead = c0 + group * size;
        const int lead_slot = 2 * lead + (group == 0 ? 1 : 0), members = min(size, c1 - lead + 1);
        if (!last_to_arrive(p.counters + lead_slot, members)) return;
        merge<D>(p, u.b, u.h, u.rt, lead_slot, 2 * lead, 1, members, groups == 1);
        if (groups == 1) return;
        if (!last_to_arrive(p.counters + 2 * (p.n_ctas * kQ4Warps) + 2 * c0 + 1, groups)) return;
        merge<D>(p, u.b, u.h, u.rt, 2 * c0 + 1, 2 * c0, size, groups, true);
    }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1) q4_attn_rows_kernel(const __grid_constant__ Q4AttnParams p) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = smem_u32(smem);
    int32_t *prefix = reinterpret_cast<int32_t *>(smem + Cfg<D>::kOffPrefix);
    Worker<D> k(p);
    k.ring = base + warp * kStages * Cfg<D>::kStageBytes;
    k.bars = base + Cfg<D>::kOffBars + warp * kStages * 8;
    k.lane = lane; k.g = lane >> 2; k.c = lane & 3;
    k.issued = k.used = 0;
    k.gave_up = false;
    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(k.bars + s * 8, 1);
        fence_mbar_init();
        fence_proxy_async();
    }
    pdl_wait();
    pdl_launch_dependents();

    // the list: prefix sums over the sequences
    List list;
    list.per_seq = p.Hkv * ((p.T * p.G + kQ4Rows - 1) / kQ4Rows);
    list.tree_tiles = (p.T + kPage - 1) / kPage;
    list.step = (p.B + kPrefix - 1) / kPrefix;
    __shared__ int warp_sum[kQ4Warps];
    int carry = 0, longest = 0;
    for (int b0 = 0; b0 < p.B; b0 += kThreads) {
        const int b = b0 + tid;
        const int L = b < p.B ? p.seq_lens[b] : 0;
        const int e = b < p.B ? entries_of(p, list, L) : 0;
        longest = max(longest, e);
        int incl = e;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += t;
        }
        __syncthreads();
        if (lane == 31) warp_sum[warp] = incl;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int i = 0; i < kQ4Warps; ++i) {
            const int x = warp_sum[i];
            before += i < warp ? x : 0;
            all += x;
        }
        if (b < p.B && b % list.step == 0) prefix[b / list.step] = carry + before + incl - e;
        carry += all;
    }
    longest = __reduce_max_sync(0xffffffffu, longest);
    __syncthreads();
    if (lane == 0) warp_sum[warp] = longest;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQ4Warps; ++i) longest = max(longest, warp_sum[i]);
    list.W = carry;
    list.n_workers = max(1, min(p.n_ctas * kQ4Warps, list.W / kMinEntries));
    // two levels of merging hold 32 x 32 shares of a unit
    longest /= list.per_seq;
    if ((int64_t)longest * list.n_workers > (int64_t)(kMaxShares - 2) * list.W)
        list.n_workers = max(1, (int)((int64_t)(kMaxShares - 2) * list.W / longest));

    // a sequence whose length cannot be: zero rows, from one block
    for (int b = blockIdx.x * kQ4Warps + warp; b < p.B; b += p.n_ctas * kQ4Warps) {
        if (length_ok(p, p.seq_lens[b])) continue;
        bool bad = false;
        for (int j = lane; j < p.T; j += 32) {
            const int a = p.parent[(size_t)b * p.T + j];
            bad |= !(j == 0 ? a == -1 : a >= 0 && a < j);
        }
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 0) p.status[b] = bad ? READER_ERR_BAD_TREE : READER_ERR_CAPACITY;
        const size_t rows = (size_t)p.T * p.Hq;
        uint4 *o = reinterpret_cast<uint4 *>(p.out + (size_t)b * rows * D);
        for (size_t i = lane; i < rows * (D / 8); i += 32) o[i] = make_uint4(0, 0, 0, 0);
        if (p.lse)
            for (size_t i = lane; i < rows; i += 32) p.lse[(size_t)b * rows + i] = 0.f;
    }

    // neighbouring ranges go to different SMs, so that few of them are spread over the GPU
    const int worker = warp * p.n_ctas + blockIdx.x;
    if (worker >= list.n_workers || list.W == 0) return;
    int w = list.begin(worker);
    const int w_end = list.begin(worker + 1);
    const uint64_t policy = l2_policy_evict_first();
    const bool once = list.per_seq == p.Hkv;   // no other unit reads these pages
    unsigned char *parents = smem + Cfg<D>::kOffParents + warp * kMaxNodes;

    Unit u;
    u.any = false;
    int flag = 0;
    for (;;) {
        // The next unit's first tiles are on their way before this one's results are written.
        Unit coming;
        int coming_flag = 0;
        coming.any = false;
        while (w < w_end && !coming.any) {
            coming = unit_at(p, list, prefix, w, w_end, lane);
            w += coming.entries;
        }
        if (coming.any && !k.gave_up) {
            if (p.num_pages == 0 && coming.t0 < coming.npages) coming_flag |= kBadPage;   // no pool to read from
            else {
                k.start(coming, coming_flag);
                for (int t = coming.t0; t < min(coming.npages, coming.t1) && t < coming.t0 + kStages; ++t)
                    k.issue(coming, t, policy, once && t >= p.shared_prefix_pages, coming_flag);
            }
        }
        if (u.any) k.finish(u, list, worker, flag);
        if (!coming.any) break;
        u = coming;
        flag = coming_flag;
        k.load_queries(u);
        k.m[0] = k.m[1] = -INFINITY;
        k.l[0] = k.l[1] = 0.f;
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) k.o[n][i] = 0.f;
        const int pages_end = p.num_pages == 0 ? u.t0 : min(u.npages, u.t1);
#pragma unroll 1
        for (int t = u.t0; t < pages_end && !k.gave_up; ++t) {
            k.await();
            if (k.gave_up) break;
            k.tile(k.ring + (k.used % kStages) * Cfg<D>::kStageBytes, min(kPage, u.L - t * kPage));
            ++k.used;
            __syncwarp();
            if (t + kStages < pages_end) k.issue(u, t + kStages, policy, once && t + kStages >= p.shared_prefix_pages, flag);
        }
        const int n0 = max(0, u.t0 - u.npages) * kPage, n1 = min(p.T, (u.t1 - u.npages) * kPage);
        if (n1 > n0) k.tree(u, n0, n1, parents, flag);
        flag = __reduce_or_sync(0xffffffffu, flag);
        if (k.gave_up || worker == p.give_up) flag |= kGaveUp;   // (the rest of the range is given up with the unit)
    }
    if (k.gave_up) {   // the block does not end under its own copies
        const uint64_t t0 = globaltimer_ns();
        for (; k.used < k.issued; ++k.used)
            while (!mbar_try_wait(k.bars + (k.used % kStages) * 8, (k.used / kStages) & 1) && globaltimer_ns() - t0 < 20000000ull) {
            }
    }
}

// Zeroes what the call counts in.
__global__ void __launch_bounds__(1024) q4_attn_zero_kernel(int4 *counters, int n, int32_t *status, int B) {
    pdl_launch_dependents();   // the attention may be set up meanwhile; it waits for this kernel's end
    pdl_wait();
    const int i = blockIdx.x * 1024 + threadIdx.x;
    if (i < n) counters[i] = make_int4(0, 0, 0, 0);
    for (int b = i; b < B; b += gridDim.x * 1024) status[b] = READER_OK;
}

}  // namespace

reader_status launch_q4_attn_rows(bool *attr_set, const Q4AttnParams &p, cudaStream_t st) {
    if (!*attr_set) {
        if (cudaFuncSetAttribute(q4_attn_rows_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<128>::kSmem) != cudaSuccess ||
            cudaFuncSetAttribute(q4_attn_rows_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<64>::kSmem) != cudaSuccess) {
            cudaGetLastError();
            return READER_ERR_CUDA;
        }
        *attr_set = true;
    }
    const int words = p.n_ctas * kQ4Warps;   // 4 counters a worker
    launch_pdl(q4_attn_zero_kernel, dim3((unsigned)((words + 1023) / 1024)), dim3(1024), 0, st, reinterpret_cast<int4 *>(p.counters), words, p.status, p.B);
    launch_pdl(p.D == 128 ? q4_attn_rows_kernel<128> : q4_attn_rows_kernel<64>, dim3((unsigned)p.n_ctas), dim3(kThreads),
               (size_t)(p.D == 128 ? Cfg<128>::kSmem : Cfg<64>::kSmem), st, p);
    return READER_OK;
}

}  // namespace reader

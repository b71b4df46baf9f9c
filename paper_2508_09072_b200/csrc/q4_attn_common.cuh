// What the kernels of the attention over a 4-bit cache share: copies, the numbers' way to bf16, the list of their work, the merge of shares.
#pragma once
#include <cfloat>

#include "ptx_sm100.cuh"
#include "q4_attn.cuh"
#include "q4_format.cuh"

namespace reader {
namespace q4 {

using namespace ptx;

constexpr float kRaiseBy = 8.f;    // log2 units by which a score may exceed the maximum in use
// The same as a difference of scores; finite whatever the scale (infinity and -inf, the maximum before the first score, have no sum).
__device__ __forceinline__ float raise_by(const Q4AttnParams &p) { return fminf(kRaiseBy / p.scale_log2, FLT_MAX); }
constexpr uint64_t kWaitLimitNs = 1000000000ull;
constexpr int kBadTree = 1, kBadLength = 2, kBadPage = 4, kGaveUp = 8;   // what is wrong with a share

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

// Whether the bf16 in the upper half of a word is an infinity or a NaN.
__device__ __forceinline__ bool nonfinite(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }
// Infinities and NaN among eight bf16 become 0; whether there was one.
__device__ __forceinline__ bool clean(uint4 &x) {
    uint32_t w[4] = {x.x, x.y, x.z, x.w}, any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= (w[i] & 0x7f807f80u) + 0x00800080u;   // (exponents of all ones carry into the sign's place)
    if (!(any & 0x80008000u)) return false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (nonfinite(w[i])) w[i] &= 0xffffu;
        if (nonfinite(w[i] << 16)) w[i] &= 0xffff0000u;
    }
    x = make_uint4(w[0], w[1], w[2], w[3]);
    return true;
}

// A pair of scales as bf16 and the pair times -24.
struct Scale2 {
    uint32_t s, m24;
};
constexpr uint32_t kScaleOne = (uint32_t)((127 - kScaleBias) << 7) * 0x10001u;
// codes: two of them, in bits 0-7 and 16-23
template <bool kWhole>
__device__ __forceinline__ Scale2 scale2(uint32_t codes) {
    Scale2 r;
    r.s = codes * 16u + kScaleOne;
    if (!kWhole) {
        if ((codes & 0xffffu) == kNanCode) r.s |= 0x7fffu;
        if ((codes >> 16) == kNanCode) r.s |= 0x7fff0000u;
    }
    r.m24 = mul_bf16x2(r.s, 0xc1c0c1c0u);
    return r;
}
// Whether a byte of the word is kNanCode: its lower seven bits carry into the eighth, and that is set.
__device__ __forceinline__ uint32_t nan_bits(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & x & 0x80808080u; }
// Pair i of a word: numbers n in the mantissas of 16 + n, times the scales, minus 24 of them: (n - 8) s, exactly.
template <int i>
__device__ __forceinline__ uint32_t pair(uint32_t w, const Scale2 &s, uint32_t sixteen) {
    const uint32_t x = i ? __funnelshift_r(w, w, 4 * i) : w;
    return fma_bf16x2((x & 0x00780078u) | sixteen, s.s, s.m24);
}

// ---- the work list
struct Unit {
    int b, h, rt, L, npages, ntiles;
    int t0, t1;              // this range's tiles
    int weight;              // entries of a tile
    int w0;                  // flat index of the unit's first entry
    int entries;             // of the flat list that this range has of the unit
    bool any;
    // the flat entry of the last tile
    __device__ __forceinline__ int last_entry(int cost) const { return w0 + cost + weight * (ntiles - 1); }
};

// The units of a KV head: n_wide of them whose tiles count `weight` entries each, and, if narrow, one more whose tiles count one.
struct List {
    int cost, pages, weight, n_wide, narrow, tree_tiles;   // entries of a unit's start and end; pages of a tile; tiles of a tree
    int step;                    // sequences per entry of the prefix table
    int W, n_workers, per_block;
    int each, more;              // entries of a range; the first `more` ranges have one more
    __device__ __forceinline__ int tiles_of(int L) const { return ((L + kPage - 1) / kPage + pages - 1) / pages + tree_tiles; }
    __device__ __forceinline__ int head_entries(int tiles) const { return n_wide * (cost + weight * tiles) + (narrow ? cost + tiles : 0); }
    __device__ __forceinline__ void cut(int workers) {
        n_workers = workers;
        each = W / workers;
        more = W - each * workers;
    }
    __device__ __forceinline__ int begin(int worker) const { return worker * each + min(worker, more); }
    // the worker whose range holds entry w
    __device__ __forceinline__ int worker_of(int w) const {
        const int longer = more * (each + 1);
        return w < longer ? w / (each + 1) : more + (w - longer) / each;
    }
};
// The sequences: for up to 32 in the lanes' registers, beyond that a table in shared memory.
struct Seqs {
    int start, L;            // of sequence `lane`
    const int2 *table;       // (start, length) of every list.step-th
};

__device__ __forceinline__ bool length_ok(const Q4AttnParams &p, int L) { return L >= 0 && (int64_t)L <= (int64_t)p.max_pages * kPage; }
__device__ __forceinline__ int entries_of(const Q4AttnParams &p, const List &l, int L) {
    return length_ok(p, L) ? p.Hkv * l.head_entries(l.tiles_of(L)) : 0;
}

// The part of the list from w on that lies in one unit (and before w_end).  Warp-collective.
__device__ __forceinline__ Unit unit_at(const Q4AttnParams &p, const List &l, const Seqs &seqs, int w, int w_end, int lane) {
    Unit u;
    int start, b;
    if (p.B <= 32) {   // the last sequence that begins at or before w (one without entries begins where the next one does)
        b = 31 - __clz(__ballot_sync(0xffffffffu, seqs.start <= w));
        start = __shfl_sync(0xffffffffu, seqs.start, b);
        u.L = __shfl_sync(0xffffffffu, seqs.L, b);
    } else {
        int lo = 0, hi = (p.B + l.step - 1) / l.step;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (seqs.table[mid].x <= w) lo = mid; else hi = mid;
        }
        const int2 x = seqs.table[lo];
        start = x.x;
        u.L = x.y;
        b = lo * l.step;
        if (l.step > 1) {   // at most 256 sequences from there on
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
    }
    u.b = b;
    u.npages = (u.L + kPage - 1) / kPage;
    u.ntiles = l.tiles_of(u.L);
    const int per_wide = l.cost + l.weight * u.ntiles, per_head = l.head_entries(u.ntiles), local = w - start;
    u.h = p.Hkv == 1 ? 0 : local / per_head;
    int pos = local - u.h * per_head, per_unit = per_wide;
    u.weight = l.weight;
    u.rt = 0;
    if (l.n_wide + l.narrow > 1) {
        u.rt = min(pos / per_wide, l.n_wide);
        pos -= u.rt * per_wide;
    }
    if (u.rt == l.n_wide) {
        u.weight = 1;
        per_unit = l.cost + u.ntiles;
    }
    const int pos_end = min(per_unit, pos + (w_end - w));
    u.entries = pos_end - pos;
    u.w0 = w - pos;
    // a tile belongs to the range that has its first entry
    u.t0 = max(0, pos - l.cost + u.weight - 1) / u.weight;
    u.t1 = max(0, pos_end - l.cost + u.weight - 1) / u.weight;
    u.any = u.t1 > u.t0;
    return u;
}

// ---- rows of a unit
// row / G (the host has checked that row * G < 2^32)
__device__ __forceinline__ int node_of(const Q4AttnParams &p, int row) { return p.G == 1 ? row : (int)__umulhi((unsigned)row, p.inv_G); }
__device__ __forceinline__ int code_of_flag(int flag) {
    return (flag & kBadTree) ? READER_ERR_BAD_TREE : (flag & kBadLength) ? READER_ERR_CAPACITY : (flag & kBadPage) ? READER_ERR_BAD_PAGE : flag ? READER_ERR_TIMEOUT : READER_OK;
}
__device__ __forceinline__ void note(const Q4AttnParams &p, int b, int flag, int lane) {
    if (flag && lane == 0) atomicMax(p.status + b, code_of_flag(flag));
}

// One row of `count` shares: ml(k) is share k's (m, l), o(k) this lane's four elements of its row of O.  A share whose maximum is -inf has weight 0 and is
// still added, so that a NaN in it stays.
struct Row {
    float top, total;
    float4 o;   // elements 4 lane .. + 3
};
template <int D, typename Ml, typename O>
__device__ __forceinline__ Row merge_row(int count, float scale_log2, const Ml &ml_of, const O &o_of) {
    const int lane = threadIdx.x & 31;
    const bool has = lane * 4 < D;
    constexpr int kAtOnce = 8;   // (this code runs once, with a cold instruction cache: 16 at once are no faster)
    Row x = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
    for (int k0 = 0; k0 < count; k0 += kAtOnce) {
        const int n = min(kAtOnce, count - k0);
        const float2 ml = lane < n ? ml_of(k0 + lane) : make_float2(-INFINITY, 0.f);
        float4 y[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            y[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (has && k < n) y[k] = o_of(k0 + k);
        }
        float top = ml.x;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        top = fmaxf(x.top, __shfl_sync(0xffffffffu, top, 0));
        const float keep = x.top == top ? 1.f : ex2((x.top - top) * scale_log2);
        const float weight = ml.x == -INFINITY ? 0.f : ml.x == top ? 1.f : ex2((ml.x - top) * scale_log2);
        float sum = ml.y * weight;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        x.top = top;
        x.total = fmaf(x.total, keep, __shfl_sync(0xffffffffu, sum, 0));
        x.o.x *= keep; x.o.y *= keep; x.o.z *= keep; x.o.w *= keep;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float w = __shfl_sync(0xffffffffu, weight, k);   // (behind the last share: 0 times 0)
            x.o.x = fmaf(y[k].x, w, x.o.x);
            x.o.y = fmaf(y[k].y, w, x.o.y);
            x.o.z = fmaf(y[k].z, w, x.o.z);
            x.o.w = fmaf(y[k].w, w, x.o.w);
        }
    }
    return x;
}
// A merged row as the call's result.
template <int D>
__device__ __forceinline__ void put_row(const Q4AttnParams &p, size_t row, const Row &x, int flag) {
    const int lane = threadIdx.x & 31;
    const float inv = x.total == 0.f ? 0.f : 1.f / x.total;   // (a row that sees nothing: zeros)
    if (lane * 4 < D)
        *reinterpret_cast<uint2 *>(p.out + row * D + lane * 4) = flag ? make_uint2(0u, 0u) : make_uint2(pack(x.o.x * inv, x.o.y * inv), pack(x.o.z * inv, x.o.w * inv));
    if (p.lse && lane == 0) p.lse[row] = flag ? 0.f : fmaf(x.top, p.scale, log2f(x.total) * 0.6931471805599453f);
}

// A row as a share in the workspace.
template <int D>
__device__ __forceinline__ void keep_row(const Q4AttnParams &p, size_t row, const Row &x) {
    const int lane = threadIdx.x & 31;
    if (lane * 4 < D) *reinterpret_cast<float4 *>(p.partial_o + row * D + lane * 4) = x.o;
    if (lane == 0) p.partial_ml[row] = make_float2(x.top, x.total);
}

// Four elements of a row of a unit, from some of its shares.
struct Part {
    float top, total;
    int flag;
    float4 x;
    // With another's added.  A part whose maximum is -inf has weight 0 and is still added, so that a NaN in it stays.
    __device__ __forceinline__ void weigh(float now, float scale_log2) {
        const float keep = top == -INFINITY ? 0.f : top == now ? 1.f : ex2((top - now) * scale_log2);
        top = now;
        total *= keep;
        x.x *= keep; x.y *= keep; x.z *= keep; x.w *= keep;
    }
    __device__ __forceinline__ void add(const Part &y, float scale_log2) {
        weigh(fmaxf(top, y.top), scale_log2);
        const float w = y.top == -INFINITY ? 0.f : y.top == top ? 1.f : ex2((y.top - top) * scale_log2);
        flag |= y.flag;
        total = fmaf(y.total, w, total);
        x.x = fmaf(y.x.x, w, x.x); x.y = fmaf(y.x.y, w, x.y); x.z = fmaf(y.x.z, w, x.z); x.w = fmaf(y.x.w, w, x.w);
    }
};
// Shares n0 .. n1 - 1 of a task, in order, by one thread; o(share) are its four elements of a share.
template <typename O>
__device__ __forceinline__ Part merge_shares(const Q4AttnParams &p, const ShareTask &t, int n0, int n1, int share_rows, int r, const O &o) {
    constexpr int kAtOnce = 4;   // shares that are read before the first is used
    Part sum = {-INFINITY, 0.f, 0, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 1
    for (int n = n0; n < n1; n += kAtOnce) {
        Part y[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            y[i] = Part{-INFINITY, 0.f, 0, make_float4(0.f, 0.f, 0.f, 0.f)};
            if (n + i < n1) {
                const int share = 2 * (t.first + n + i) + (n + i == 0 ? 1 : 0);
                const float2 ml = p.partial_ml[(size_t)share * share_rows + r];
                y[i] = Part{ml.x, ml.y, p.flags[share], o(share)};
            }
        }
        float now = sum.top;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) now = fmaxf(now, y[i].top);
        sum.weigh(now, p.scale_log2);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const float w = y[i].top == -INFINITY ? 0.f : y[i].top == now ? 1.f : ex2((y[i].top - now) * p.scale_log2);
            sum.flag |= y[i].flag;
            sum.total = fmaf(y[i].total, w, sum.total);
            sum.x.x = fmaf(y[i].x.x, w, sum.x.x); sum.x.y = fmaf(y[i].x.y, w, sum.x.y);
            sum.x.z = fmaf(y[i].x.z, w, sum.x.z); sum.x.w = fmaf(y[i].x.w, w, sum.x.w);
        }
    }
    return sum;
}
// The call's result: elements 4 c .. + 3 of row r of a task's unit.
template <int D>
__device__ __forceinline__ void put_merged(const Q4AttnParams &p, const ShareTask &t, int unit_rows, int r, int c, const Part &y) {
    const int g = t.rt * unit_rows + r, j = node_of(p, g);
    const size_t row = ((size_t)t.b * p.T + j) * p.Hq + t.h * p.G + (g - j * p.G);
    const float inv = y.total == 0.f ? 0.f : 1.f / y.total;   // (a row that sees nothing: zeros)
    *reinterpret_cast<uint2 *>(p.out + row * D + c * 4) = y.flag ? make_uint2(0u, 0u) : make_uint2(pack(y.x.x * inv, y.x.y * inv), pack(y.x.z * inv, y.x.w * inv));
    if (c != 0) return;
    if (p.lse) p.lse[row] = y.flag ? 0.f : fmaf(y.top, p.scale, log2f(y.total) * 0.6931471805599453f);
    if (r == 0) note(p, t.b, y.flag, 0);
}

// Whether parent array b is a tree.  Warp-collective.
__device__ __forceinline__ bool tree_ok(const Q4AttnParams &p, int b, int lane) {
    bool bad = false;
    for (int j = lane; j < p.T; j += 32) {
        const int a = p.parent[(size_t)b * p.T + j];
        bad |= !(j == 0 ? a == -1 : a >= 0 && a < j);
    }
    return !__any_sync(0xffffffffu, bad);
}


// Sequences whose length cannot be: zero rows and their status word, a warp `me` of `warps` for each.
template <int D>
__device__ __forceinline__ void reject_lengths(const Q4AttnParams &p, int me, int warps, int lane) {
    for (int b = me; b < p.B; b += warps) {
        if (length_ok(p, p.seq_lens[b])) continue;
        const bool tree = tree_ok(p, b, lane);
        if (lane == 0) p.status[b] = tree ? READER_ERR_CAPACITY : READER_ERR_BAD_TREE;
        const size_t rows = (size_t)p.T * p.Hq;
        uint4 *o = reinterpret_cast<uint4 *>(p.out + (size_t)b * rows * D);
        for (size_t i = lane; i < rows * (D / 8); i += 32) o[i] = make_uint4(0, 0, 0, 0);
        if (p.lse)
            for (size_t i = lane; i < rows; i += 32) p.lse[(size_t)b * rows + i] = 0.f;
    }
}

// The list of a call: prefix sums over the sequences, by every warp itself for up to 32, else by the thread block with a table of kPrefix
// entries in shared memory.  warp_sum: one word per warp.  Block-collective; ends without a barrier.
constexpr int kPrefix = 256;
template <int kWarps>
__device__ __forceinline__ void make_list(const Q4AttnParams &p, List &list, Seqs &seqs, int2 *table, int *warp_sum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    list.step = (p.B + kPrefix - 1) / kPrefix;
    seqs.table = table;
    seqs.start = 0x7fffffff;
    seqs.L = 0;
    list.W = 0;
    if (p.B <= 32) {
        const int L = lane < p.B ? p.seq_lens[lane] : -1, e = lane < p.B ? entries_of(p, list, L) : 0;
        int incl = e;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += t;
        }
        if (lane < p.B) seqs.start = incl - e;
        seqs.L = L;
        list.W = __shfl_sync(0xffffffffu, incl, 31);
        return;
    }
    for (int b0 = 0; b0 < p.B; b0 += kWarps * 32) {
        const int b = b0 + tid;
        const int L = b < p.B ? p.seq_lens[b] : 0;
        const int e = b < p.B ? entries_of(p, list, L) : 0;
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
        for (int i = 0; i < kWarps; ++i) {
            const int x = warp_sum[i];
            before += i < warp ? x : 0;
            all += x;
        }
        if (b < p.B && b % list.step == 0) table[b / list.step] = make_int2(list.W + before + incl - e, L);
        list.W += all;
    }
}

}  // namespace q4
}  // namespace reader

// From a projection's output to the operands of attention (reader_prompt_append, reader_tree_rotate): every query
// and key head is normalised, y = x rsqrt(mean(x^2) + eps) w, and rotated by its token's position, in one pass;
// keys and values go to their place (a page of the cache, or the tree tensors), queries to a dense tensor.
//
// Rotation of a pair (a, b) by the table row (cos, sin) of the position: (a cos - b sin, b cos + a sin).  The pairs
// are (j, j + R/2) of the first R = rot_dim elements, or (2j, 2j + 1) when interleaved.
//
// Bound: bytes.  A head row is read once and written once, 2 (Hq + 2 Hkv) D bf16 per token; all arithmetic is fp32
// on values that stay in registers, with one rounding to bf16 at the very end.  D/8 neighbouring threads hold a head,
// each of them the four elements of a first half and the four partners they are rotated with (two 8-byte accesses),
// so the rotation needs no exchange and the mean square a few shuffles.  A warp walks the heads of one token by
// itself (or a share of them, when there are too few tokens to fill the GPU), with several accesses under way and the
// token's table row in registers; its rows are asked for (an L2 prefetch) before it finds out
// which sequence the token belongs to and where it goes.
#include "common.cuh"
#include "rotate.cuh"

namespace reader {
namespace {

// Small blocks: a block's registers are free for the next one when its slowest warp is done (256 threads, 64 x 128 nodes:
// 40.7 us, 128 threads: 40.0).
constexpr int kThreads = 128;
constexpr int kInFlight = 4;   // head rows a thread has under way (two accesses each)

__device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack(float2 x) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
    return *reinterpret_cast<const uint32_t *>(&h);
}

struct Raw {
    uint2 a, b;   // four elements each
};

// A thread's part of a head: which elements it has, and its table entries.
//   half-split (kInter false): word i of a and word i of b are two pairs as they stand
//   interleaved: (a0 a1), (b0 b1) are the pairs; the even elements (a0 b0) are brought into one word, the odd ones into the other
template <int D, bool kInter>
struct Turner {
    static constexpr int kLanes = D / 8;   // threads per head
    int ea, eb;            // where its two groups of four elements begin
    int at;                // its four pairs' index in the table; -1: its elements are not rotated
    float2 c[2], s[2];

    __device__ __forceinline__ void init(const RotateParams &p, int lane) {
        const int l = lane % kLanes, quads = p.rope ? p.rot / 8 : 0;   // threads with rotated elements
        const bool turned = l < quads, halves = turned && !kInter;
        at = turned ? 4 * l : -1;
        ea = halves ? 4 * l : 8 * l;       // (behind the rotated threads the rest of the head, 8 elements each)
        eb = halves ? ea + p.rot / 2 : ea + 4;
    }
    // first elements of the pairs to .a, second ones to .b (its own inverse)
    static __device__ __forceinline__ Raw paired(const Raw &r) {
        if (!kInter) return r;
        return Raw{make_uint2(__byte_perm(r.a.x, r.b.x, 0x5410), __byte_perm(r.a.y, r.b.y, 0x5410)),
                   make_uint2(__byte_perm(r.a.x, r.b.x, 0x7632), __byte_perm(r.a.y, r.b.y, 0x7632))};
    }
    __device__ __forceinline__ void load_table(const RotateParams &p, int64_t pos) {
        if (at < 0) return;
        const float *row = p.rope + pos * p.rot + at;
        const float4 x = *reinterpret_cast<const float4 *>(row), y = *reinterpret_cast<const float4 *>(row + p.rot / 2);
        // pairs 0 .. 3 in the order of the words: (0 1), (2 3), or (0 2), (1 3) when interleaved
        c[0] = make_float2(x.x, kInter ? x.z : x.y); c[1] = make_float2(kInter ? x.y : x.z, x.w);
        s[0] = make_float2(y.x, kInter ? y.z : y.y); s[1] = make_float2(kInter ? y.y : y.z, y.w);
    }
};

// What one kind of heads (queries or keys) is multiplied with: the table entries and the norm's weights in one.
template <int D, bool kInter>
struct Factors {
    float2 ac[2], bs[2], bc[2], as[2];   // first elements by cos, second ones by -sin; second ones by cos, first ones by sin
    __device__ __forceinline__ void init(const RotateParams &p, const Turner<D, kInter> &t, const __nv_bfloat16 *weight) {
        float2 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = make_float2(1.f, 1.f);
        if (p.q_weight) {
            const Raw r = t.paired(Raw{*reinterpret_cast<const uint2 *>(weight + t.ea), *reinterpret_cast<const uint2 *>(weight + t.eb)});
            w[0] = unpack(r.a.x); w[1] = unpack(r.a.y); w[2] = unpack(r.b.x); w[3] = unpack(r.b.y);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (t.at >= 0) {
                ac[i] = __fmul2_rn(w[i], t.c[i]);
                bs[i] = __fmul2_rn(w[i + 2], make_float2(-t.s[i].x, -t.s[i].y));
                bc[i] = __fmul2_rn(w[i + 2], t.c[i]);
                as[i] = __fmul2_rn(w[i], t.s[i]);
            } else {
                ac[i] = w[i];
                bc[i] = w[i + 2];
                bs[i] = as[i] = make_float2(0.f, 0.f);
            }
        }
    }
    // Warp-collective (all heads of a warp at once).
    __device__ __forceinline__ Raw turn(const RotateParams &p, const Turner<D, kInter> &t, const Raw &raw) const {
        const Raw r = t.paired(raw);
        const float2 a[2] = {unpack(r.a.x), unpack(r.a.y)}, b[2] = {unpack(r.b.x), unpack(r.b.y)};
        float2 y[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            y[i] = __fmul2_rn(a[i], ac[i]);
            y[i + 2] = __fmul2_rn(b[i], bc[i]);
            if (t.at >= 0) {   // (not by a factor of zero: the other element may be infinite)
                y[i] = __ffma2_rn(b[i], bs[i], y[i]);
                y[i + 2] = __ffma2_rn(a[i], as[i], y[i + 2]);
            }
        }
        if (p.q_weight) {
            float2 sq = __fmul2_rn(a[0], a[0]);
            sq = __ffma2_rn(a[1], a[1], sq);
            sq = __ffma2_rn(b[0], b[0], sq);
            sq = __ffma2_rn(b[1], b[1], sq);
            float ss = sq.x + sq.y;
#pragma unroll
            for (int d = Turner<D, kInter>::kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
            const float f = rsqrtf(ss * (1.f / D) + p.eps);
            const float2 f2 = make_float2(f, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = __fmul2_rn(y[i], f2);
        }
        return t.paired(Raw{make_uint2(pack(y[0]), pack(y[1])), make_uint2(pack(y[2]), pack(y[3]))});
    }
};

// One kind of a token's heads (queries, keys or values): from `src` to `dst`, where heads are kStride elements apart.
// A warp handles 32 / kLanes heads at once and takes every `share`-th such group, from group `first`; kInFlight of
// them are loaded before the first is worked on.  kShare 1: all groups, at offsets known to the compiler.
template <int D, bool kInter, int kShare, int kStride, bool kTurn>
__device__ __forceinline__ void walk_heads(const RotateParams &p, const Turner<D, kInter> &t, const __nv_bfloat16 *src, __nv_bfloat16 *dst, int heads,
                                           int first, const __nv_bfloat16 *weight) {
    constexpr int kGroup = 32 / Turner<D, kInter>::kLanes;
    const int sub = (threadIdx.x & 31) / Turner<D, kInter>::kLanes, step = kShare == 1 ? kGroup : kGroup * p.share;
    Factors<D, kInter> by;
    if (kTurn) by.init(p, t, weight);
    int x = first * kGroup + sub;
    const __nv_bfloat16 *sa = src + x * D + t.ea, *sb = src + x * D + t.eb;
    __nv_bfloat16 *da = dst + (size_t)x * kStride + t.ea, *db = dst + (size_t)x * kStride + t.eb;
    for (; x - sub + step * (kInFlight - 1) + kGroup <= heads; x += step * kInFlight) {
        Raw raw[kInFlight];
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            raw[i].a = *reinterpret_cast<const uint2 *>(sa + i * step * D);
            raw[i].b = *reinterpret_cast<const uint2 *>(sb + i * step * D);
        }
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            const Raw y = kTurn ? by.turn(p, t, raw[i]) : raw[i];
            *reinterpret_cast<uint2 *>(da + (size_t)(i * step) * kStride) = y.a;
            *reinterpret_cast<uint2 *>(db + (size_t)(i * step) * kStride) = y.b;
        }
        sa += kInFlight * step * D;
        sb += kInFlight * step * D;
        da += (size_t)(kInFlight * step) * kStride;
        db += (size_t)(kInFlight * step) * kStride;
    }
#pragma unroll 1
    for (; x - sub < heads; x += step) {   // the last few groups, the very last perhaps not whole
        Raw raw{};
        if (x < heads) {
            raw.a = *reinterpret_cast<const uint2 *>(sa);
            raw.b = *reinterpret_cast<const uint2 *>(sb);
        }
        const Raw y = kTurn ? by.turn(p, t, raw) : raw;
        if (x < heads) {
            *reinterpret_cast<uint2 *>(da) = y.a;
            *reinterpret_cast<uint2 *>(db) = y.b;
        }
        sa += step * D;
        sb += step * D;
        da += (size_t)step * kStride;
        db += (size_t)step * kStride;
    }
}

// A token's heads as this warp has them: every p.share-th group of all heads, queries first, then keys, then values.
template <int D, bool kInter, int kShare>
struct Token {
    static constexpr int kGroup = 32 / Turner<D, kInter>::kLanes;
    const __nv_bfloat16 *q, *k, *v;
    int q_first, k_first, v_first;   // this warp's first group of each kind

    __device__ __forceinline__ void init(const RotateParams &p, int64_t row, int first) {
        q = p.q + row * p.q_stride;
        k = p.k + row * p.k_stride;
        v = p.v + row * p.v_stride;
        const int q_groups = (p.Hq + kGroup - 1) / kGroup, kv_groups = (p.Hkv + kGroup - 1) / kGroup, mask = p.share - 1;
        q_first = first;
        k_first = (first - q_groups) & mask;
        v_first = (first - q_groups - kv_groups) & mask;
    }
    // Asks for the warp's rows (its first ones, if it has but a share of them), so that they are under way while it finds
    // out where they go.
    __device__ __forceinline__ void prefetch(const RotateParams &p, const Turner<D, kInter> &t, int lane) const {
        auto ask = [&](const __nv_bfloat16 *at) { asm volatile("prefetch.global.L2 [%0];" ::"l"(at)); };
        if (kShare == 1) {
            for (int i = lane * 64; i < p.Hq * D; i += 32 * 64) ask(q + i);
            for (int i = lane * 64; i < p.Hkv * D; i += 32 * 64) {
                ask(k + i);
                ask(v + i);
            }
            return;
        }
        const int sub = lane / Turner<D, kInter>::kLanes;
        auto ask_head = [&](const __nv_bfloat16 *head) {
            ask(head + t.ea);
            if (t.eb - t.ea >= 64) ask(head + t.eb);
        };
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int x = (q_first + i * p.share) * kGroup + sub;
            if (x < p.Hq) ask_head(q + x * D);
        }
        if (k_first * kGroup + sub < p.Hkv) ask_head(k + (k_first * kGroup + sub) * D);
        if (v_first * kGroup + sub < p.Hkv) ask_head(v + (v_first * kGroup + sub) * D);
    }
    template <int kStride>
    __device__ __forceinline__ void move(const RotateParams &p, const Turner<D, kInter> &t, __nv_bfloat16 *q_dst, __nv_bfloat16 *k_dst,
                                         __nv_bfloat16 *v_dst) const {
        walk_heads<D, kInter, kShare, D, true>(p, t, q, q_dst, p.Hq, q_first, p.q_weight);
        walk_heads<D, kInter, kShare, kStride, true>(p, t, k, k_dst, p.Hkv, k_first, p.k_weight);
        walk_heads<D, kInter, kShare, kStride, false>(p, t, v, v_dst, p.Hkv, v_first, nullptr);
    }
};

// Zeros in place of a warp's share of a rejected token's heads (all warps of the token together: all of it).
template <int D>
__device__ __forceinline__ void zero_heads(__nv_bfloat16 *dst, int heads, int first, int share, int lane) {
    for (int i = first * 32 + lane; i < heads * (D / 8); i += share * 32) reinterpret_cast<uint4 *>(dst)[i] = make_uint4(0, 0, 0, 0);
}

// What keeps sequence b's n new tokens from being written.  Warp-collective.
__device__ __forceinline__ int append_status(const RotateParams &p, int b, int n, int L, int lane) {
    if (n == 0) return L < 0 ? READER_ERR_CAPACITY : READER_OK;
    bool room = L >= 0 && L >= p.shared_prefix_len && (int64_t)L + n <= (int64_t)p.max_pages * kPage;
    if (p.rope && (int64_t)L + n > p.max_positions) room = false;
    if (!room) return READER_ERR_CAPACITY;
    bool bad = false;
    for (int i = L / kPage + lane; i <= (L + n - 1) / kPage; i += 32) {
        const int pg = p.page_table[(size_t)b * p.max_pages + i];
        bad |= pg < 0 || pg >= p.num_pages;
    }
    return __any_sync(0xffffffffu, bad) ? READER_ERR_BAD_PAGE : READER_OK;
}

// Warps 0 .. tokens * share - 1: one token's heads, or a share of them.  Warps behind them: one sequence's status
// word each.
// Every warp looks through token_start for its token's sequence and through the pages that the sequence's new tokens take.  That
// is nothing for batches of some hundreds and prompts of some ten thousand tokens, and more than the rows beyond: single tokens
// (32/8/128) of 1024, 8192, 32768 sequences 10, 75, 833 us (rows alone: 3.9, 31, 125), one prompt (4/1/128) of 16 k, 128 k,
// 512 k tokens 17.5, 170, 1315 us (7.8, 62, 249).
template <int D, bool kInter, int kShare>
__global__ void __launch_bounds__(kThreads, 6) prompt_append_kernel(const RotateParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int share = kShare == 1 ? 1 : p.share;
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), writers = (int64_t)p.tokens * share;
    const int token = w < writers ? (int)(w / share) : -1;
    if (w >= writers + p.B) return;
    // One pass over token_start: is it in order, and whose token is this (-1: nobody's)?
    int start = 0, n = 0;
    auto owner = [&]() -> int {
        bool bad = false;
        int mine = -1;
        for (int i = lane; i < p.B; i += 32) {
            const int a = p.token_start[i], e = p.token_start[i + 1];
            bad |= a < 0 || a > e || e > p.tokens;
            if (token >= 0 && a <= token && token < e) mine = i;
        }
        if (__any_sync(0xffffffffu, bad)) return -2;
        const int b = token >= 0 ? __reduce_max_sync(0xffffffffu, mine) : (int)(w - writers);
        if (b < 0) return -1;
        start = p.token_start[b];
        n = p.token_start[b + 1] - start;
        return b;
    };
    if (token < 0) {
        const int b = owner();
        const int st = b == -2 ? READER_ERR_INVALID_ARG : append_status(p, b, n, p.seq_lens[b], lane);
        if (lane == 0) p.status[w - writers] = st;
        return;
    }
    Turner<D, kInter> t;
    t.init(p, lane);
    const int first = (int)(w % share);
    Token<D, kInter, kShare> tok;
    tok.init(p, token, first);
    tok.prefetch(p, t, lane);
    const int b = owner();
    if (b < 0) return;
    __nv_bfloat16 *q_row = p.q_out + (size_t)token * p.Hq * D;
    const int L = p.seq_lens[b];
    if (append_status(p, b, n, L, lane) != READER_OK) return zero_heads<D>(q_row, p.Hq, first, share, lane);
    const int pos = L + (token - start);
    t.load_table(p, pos);
    const int page = p.page_table[(size_t)b * p.max_pages + pos / kPage];
    const size_t at = ((size_t)page * p.Hkv * kPage + pos % kPage) * D;
    tok.template move<kPage * D>(p, t, q_row, p.k_out + at, p.v_out + at);
}

// Block (y, b): the warps y * 4 .. y * 4 + 3 of sequence b; warp j * share + s: node j of its tree, or a share of its heads.
template <int D, bool kInter, int kShare>
__global__ void __launch_bounds__(kThreads, 6) tree_rotate_kernel(const RotateParams p) {
    __shared__ int32_t par[kMaxNodes];
    pdl_wait();
    pdl_launch_dependents();
    const int share = kShare == 1 ? 1 : p.share, lane = threadIdx.x & 31, blocks = (p.T * share + kThreads / 32 - 1) / (kThreads / 32);
    const int b = blockIdx.x / blocks, w = (blockIdx.x - b * blocks) * (kThreads / 32) + (threadIdx.x >> 5);
    const int j = w / share, first = w - j * share;
    const int64_t row = (int64_t)b * p.T + min(j, p.T - 1);
    Turner<D, kInter> t;
    t.init(p, lane);
    Token<D, kInter, kShare> tok;
    tok.init(p, row, first);
    tok.prefetch(p, t, lane);
    const int L = p.seq_lens[b];
    bool bad = false;
    for (int i = threadIdx.x; i < p.T; i += kThreads) {
        const int above = p.parent[(size_t)b * p.T + i];
        bad |= !(i == 0 ? above == -1 : above >= 0 && above < i);
        par[i] = above;
    }
    const bool bad_tree = __syncthreads_or(bad);
    if (j >= p.T) return;
    auto nodes_above = [&](int i) {   // the chain strictly decreases on a valid tree
        int n = 0;
        for (i = par[i]; i >= 0; i = par[i]) ++n;
        return n;
    };
    bool no_room = L < 0;
    // only a table that might be too short needs every node's depth
    if (p.rope && !bad_tree && (int64_t)L + p.T > p.max_positions) {
        for (int i = lane; i < p.T; i += 32) no_room |= (int64_t)L + nodes_above(i) >= p.max_positions;
        no_room = __any_sync(0xffffffffu, no_room);
    }
    if (j == 0 && first == 0 && lane == 0) p.status[b] = bad_tree ? READER_ERR_BAD_TREE : no_room ? READER_ERR_CAPACITY : READER_OK;
    __nv_bfloat16 *q_row = p.q_out + row * p.Hq * D, *k_row = p.k_out + row * p.Hkv * D, *v_row = p.v_out + row * p.Hkv * D;
    if (bad_tree || no_room) {
        zero_heads<D>(q_row, p.Hq, first, p.share, lane);
        zero_heads<D>(k_row, p.Hkv, first, p.share, lane);
        zero_heads<D>(v_row, p.Hkv, first, p.share, lane);
        return;
    }
    t.load_table(p, (int64_t)L + nodes_above(j));
    tok.template move<D>(p, t, q_row, k_row, v_row);
}

// Warps per token: one, unless that leaves the GPU short of warps (16 an SM); a power of two, at most the first that gives every
// group of heads a warp of its own (32/8/128 heads are 24 groups: up to 32 warps, 8 of them without a head).
int warps_per_token(int64_t tokens, int heads, int D, int n_sm) {
    const int groups = (heads * (D / 8) + 31) / 32;
    int share = 1;
    while (share < groups && tokens * share < 16 * (int64_t)n_sm) share *= 2;
    return share;
}
dim3 blocks_for(int64_t warps) { return dim3((unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32))); }

}  // namespace

// The kernel for the head dimension, the kind of pairs and whether tokens are shared among warps.
#define ROTATE_KERNEL(name, p)                                                                                               \
    ((p).D == 128 ? ((p).interleaved ? ((p).share == 1 ? name<128, true, 1> : name<128, true, 0>)                           \
                                     : ((p).share == 1 ? name<128, false, 1> : name<128, false, 0>))                        \
                  : ((p).interleaved ? ((p).share == 1 ? name<64, true, 1> : name<64, true, 0>)                             \
                                     : ((p).share == 1 ? name<64, false, 1> : name<64, false, 0>)))

void launch_prompt_append(RotateParams p, int n_sm, cudaStream_t st) {
    p.share = warps_per_token(p.tokens, p.Hq + 2 * p.Hkv, p.D, n_sm);
    launch_pdl(ROTATE_KERNEL(prompt_append_kernel, p), blocks_for((int64_t)p.tokens * p.share + p.B), dim3(kThreads), 0, st, p);
}

void launch_tree_rotate(RotateParams p, int n_sm, cudaStream_t st) {
    p.share = warps_per_token((int64_t)p.B * p.T, p.Hq + 2 * p.Hkv, p.D, n_sm);
    const int per_seq = (p.T * p.share + kThreads / 32 - 1) / (kThreads / 32);
    launch_pdl(ROTATE_KERNEL(tree_rotate_kernel, p), dim3((unsigned)(p.B * per_seq)), dim3(kThreads), 0, st, p);
}

}  // namespace reader

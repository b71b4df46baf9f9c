// From a projection's output to the operands of attention (reader_prompt_append, reader_tree_rotate): every query
// and key head is normalised, y = x rsqrt(mean(x^2) + eps) w, and rotated by its token's position, in one pass;
// keys and values go to their place (a page of the cache, or the tree tensors), queries to a dense tensor.
//
// Rotation of a pair (a, b) by the table row (cos, sin) of the position: (a cos - b sin, b cos + a sin).  The pairs
// are (j, j + R/2) of the first R = rot_dim elements, or (2j, 2j + 1) when interleaved.
//
// Bound: bytes.  A head row is read once and written once, 2 (Hq + 2 Hkv) D bf16 per token; all arithmetic is fp32
// on values that stay in registers, with one rounding to bf16 at the very end.  One block per token: a thread holds
// eight consecutive elements (one 16-byte access) of one head, D/8 neighbouring threads hold a head, so the mean
// square is a few shuffles, the half-split partner is one shuffle away and the table row is read once per thread
// for all of its heads.  The loads of the head rows are issued before the block finds out which sequence its token
// belongs to and where it goes.
#include "common.cuh"
#include "rotate.cuh"

namespace reader {
namespace {

constexpr int kThreads = 256;
constexpr int kInFlight = 4;   // head rows a thread loads before it works on the first

struct Row8 {
    float x[8];
};

__device__ __forceinline__ Row8 unpack(const uint4 &raw) {
    Row8 r;
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.x[2 * i] = __uint_as_float(w[i] << 16);
        r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    return r;
}
__device__ __forceinline__ uint4 pack(const Row8 &r) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(r.x[2 * i], r.x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The token-independent part of a thread's work: its eight elements' weights and their table entries.
template <int D>
struct Turner {
    static constexpr int kLanes = D / 8;   // threads per head
    int l;                // this thread's place in its head
    int src_lane;         // half-split: the lane of the partner elements
    int mode;             // 0: elements pass unrotated, 1: first half of a half-split pair, 2: second half, 3: interleaved
    float c[8], s[8];
    uint4 wq, wk;

    __device__ __forceinline__ void init(const RotateParams &p, int lane) {
        l = lane % kLanes;
        src_lane = lane;
        mode = 0;
        if (p.q_weight) {
            wq = reinterpret_cast<const uint4 *>(p.q_weight)[l];
            wk = reinterpret_cast<const uint4 *>(p.k_weight)[l];
        }
        if (p.rope && l * 8 < p.rot) {
            const int half8 = p.rot / 16;   // threads per half
            if (p.interleaved) {
                mode = 3;
            } else {
                mode = l < half8 ? 1 : 2;
                src_lane = mode == 1 ? lane + half8 : lane - half8;
            }
        }
    }
    __device__ __forceinline__ void load_table(const RotateParams &p, int64_t pos) {
        if (mode == 0) return;
        const int half = p.rot / 2;
        const float *row = p.rope + pos * p.rot;
        if (mode == 3) {
            const float4 a = *reinterpret_cast<const float4 *>(row + 4 * l), b = *reinterpret_cast<const float4 *>(row + half + 4 * l);
            c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w;
            s[0] = b.x; s[1] = b.y; s[2] = b.z; s[3] = b.w;
        } else {
            const int at = 8 * l - (mode == 2 ? half : 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 a = *reinterpret_cast<const float4 *>(row + at + 4 * i), b = *reinterpret_cast<const float4 *>(row + half + at + 4 * i);
                c[4 * i] = a.x; c[4 * i + 1] = a.y; c[4 * i + 2] = a.z; c[4 * i + 3] = a.w;
                s[4 * i] = b.x; s[4 * i + 1] = b.y; s[4 * i + 2] = b.z; s[4 * i + 3] = b.w;
            }
        }
    }
    // Warp-collective (all heads of a warp at once).
    __device__ __forceinline__ uint4 turn(const RotateParams &p, const uint4 &raw, bool key) const {
        Row8 r = unpack(raw);
        if (p.q_weight) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(r.x[i], r.x[i], ss);
#pragma unroll
            for (int d = kLanes / 2; d > 0; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
            const float f = rsqrtf(ss * (1.f / D) + p.eps);
            const Row8 w = unpack(key ? wk : wq);
#pragma unroll
            for (int i = 0; i < 8; ++i) r.x[i] = r.x[i] * f * w.x[i];
        }
        if (p.rope) {
            if (p.interleaved) {
                if (mode == 3) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = r.x[2 * i], b = r.x[2 * i + 1];
                        r.x[2 * i] = a * c[i] - b * s[i];
                        r.x[2 * i + 1] = b * c[i] + a * s[i];
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float o = __shfl_sync(0xffffffffu, r.x[i], src_lane);
                    if (mode == 1) r.x[i] = r.x[i] * c[i] - o * s[i];
                    else if (mode == 2) r.x[i] = r.x[i] * c[i] + o * s[i];
                }
            }
        }
        return pack(r);
    }
};

// All head rows of one token: `row` is its row of the projection's output.  place(x, l) gives where piece l of
// output head x goes (queries first, then keys, then values); `known()` runs once, after the first loads are in
// flight, and says whether the token is written (1), zeroed (0) or left alone (-1).
template <int D, typename Known, typename Place>
__device__ __forceinline__ void token_heads(const RotateParams &p, int64_t row, Turner<D> &t, const Known &known, const Place &place) {
    constexpr int kLanes = D / 8, kPass = kThreads / kLanes;
    const int heads = p.Hq + 2 * p.Hkv, slot = threadIdx.x / kLanes;
    const __nv_bfloat16 *q = p.q + row * p.q_stride, *k = p.k + row * p.k_stride, *v = p.v + row * p.v_stride;
    int what = 1;
    for (int x0 = 0; x0 < heads; x0 += kPass * kInFlight) {
        uint4 raw[kInFlight];
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            const int x = x0 + i * kPass + slot;
            raw[i] = make_uint4(0, 0, 0, 0);
            if (x < heads) {
                const __nv_bfloat16 *src = x < p.Hq ? q + (size_t)x * D : x < p.Hq + p.Hkv ? k + (size_t)(x - p.Hq) * D : v + (size_t)(x - p.Hq - p.Hkv) * D;
                raw[i] = reinterpret_cast<const uint4 *>(src)[t.l];
            }
        }
        if (x0 == 0) {
            what = known();
            if (what < 0) return;
        }
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            if (x0 + i * kPass >= heads) break;   // (the same for the whole block)
            const int x = x0 + i * kPass + slot;
            const uint4 turned = t.turn(p, raw[i], x >= p.Hq);
            uint4 y = x < p.Hq + p.Hkv ? turned : raw[i];
            if (what == 0) y = make_uint4(0, 0, 0, 0);
            if (x < heads)
                if (uint4 *dst = place(x)) dst[t.l] = y;
        }
    }
}

// What is wrong with sequence b of a prompt whose pair (first, last) of token_start is in order; block-wide.
__device__ __forceinline__ int append_status(const RotateParams &p, int b, int n) {
    const int L = p.seq_lens[b];
    bool room = L >= 0 && L >= p.shared_prefix_len && (int64_t)L + n <= (int64_t)p.max_pages * kPage;
    if (p.rope && (int64_t)L + n > p.max_positions) room = false;
    if (n == 0) return L < 0 ? READER_ERR_CAPACITY : READER_OK;
    if (!room) return READER_ERR_CAPACITY;
    bool bad = false;
    for (int i = L / kPage + threadIdx.x; i <= (L + n - 1) / kPage; i += blockDim.x) {
        const int pg = p.page_table[(size_t)b * p.max_pages + i];
        bad |= pg < 0 || pg >= p.num_pages;
    }
    return __syncthreads_or(bad) ? READER_ERR_BAD_PAGE : READER_OK;
}

// Blocks 0 .. total_tokens-1: one token each.  Blocks behind them: one sequence's status word each.
template <int D>
__global__ void __launch_bounds__(kThreads) prompt_append_kernel(const RotateParams p) {
    __shared__ int s_seq;
    pdl_wait();
    pdl_launch_dependents();
    const int token = blockIdx.x < (unsigned)p.tokens ? (int)blockIdx.x : -1;
    // One pass over token_start: is it in order, and whose token is this?  Block-wide; -1: nobody's.
    auto owner = [&](int &start, int &n) -> int {
        if (threadIdx.x == 0) s_seq = -1;
        __syncthreads();
        bool bad = false;
        for (int i = threadIdx.x; i < p.B; i += kThreads) {
            const int a = p.token_start[i], e = p.token_start[i + 1];
            bad |= a < 0 || a > e || e > p.tokens;
            if (token >= 0 && a <= token && token < e) s_seq = i;
        }
        if (__syncthreads_or(bad)) return -2;
        const int b = token >= 0 ? s_seq : (int)blockIdx.x - p.tokens;
        if (b < 0) return -1;
        start = p.token_start[b];
        n = p.token_start[b + 1] - start;
        return b;
    };
    int start = 0, n = 0;
    if (token < 0) {
        const int b = owner(start, n);
        const int st = b == -2 ? READER_ERR_INVALID_ARG : append_status(p, b, n);
        if (threadIdx.x == 0) p.status[blockIdx.x - p.tokens] = st;
        return;
    }
    Turner<D> t;
    t.init(p, threadIdx.x & 31);
    uint4 *k_dst = nullptr, *v_dst = nullptr;
    token_heads<D>(
        p, token, t,
        [&]() {
            const int b = owner(start, n);
            if (b < 0) return -1;
            if (append_status(p, b, n) != READER_OK) return 0;
            const int pos = p.seq_lens[b] + (token - start);
            const int page = p.page_table[(size_t)b * p.max_pages + pos / kPage];
            const size_t at = ((size_t)page * p.Hkv * kPage + pos % kPage) * D;
            k_dst = reinterpret_cast<uint4 *>(p.k_out + at);
            v_dst = reinterpret_cast<uint4 *>(p.v_out + at);
            t.load_table(p, pos);
            return 1;
        },
        [&](int x) -> uint4 * {
            constexpr size_t kHeadPieces = (size_t)kPage * D / 8;
            if (x < p.Hq) return reinterpret_cast<uint4 *>(p.q_out + ((size_t)token * p.Hq + x) * D);
            if (!k_dst) return nullptr;
            return x < p.Hq + p.Hkv ? k_dst + (x - p.Hq) * kHeadPieces : v_dst + (x - p.Hq - p.Hkv) * kHeadPieces;
        });
}

// Block b * T + j: node j of sequence b's tree.
template <int D>
__global__ void __launch_bounds__(kThreads) tree_rotate_kernel(const RotateParams p) {
    __shared__ int hop[2][kMaxNodes + 1], depth[2][kMaxNodes + 1];
    pdl_wait();
    pdl_launch_dependents();
    const int b = blockIdx.x / p.T, j = blockIdx.x - b * p.T, tid = threadIdx.x;
    const int64_t row = blockIdx.x;
    Turner<D> t;
    t.init(p, tid & 31);
    token_heads<D>(
        p, row, t,
        [&]() {
            // depth of every node by doubling: after step i, hop is the ancestor 2^i levels up (T: above the root) and
            // depth the nodes passed on the way
            bool bad = false;
            for (int i = tid; i <= p.T; i += kThreads) {
                const int par = i < p.T ? p.parent[(size_t)b * p.T + i] : -1;
                const bool ok = i == p.T || (i == 0 ? par == -1 : par >= 0 && par < i);
                bad |= !ok;
                hop[0][i] = ok && par >= 0 ? par : p.T;
                depth[0][i] = i < p.T;
            }
            const bool bad_tree = __syncthreads_or(bad);
            int cur = 0;
            for (int step = 1; step < p.T; step <<= 1) {
                for (int i = tid; i <= p.T; i += kThreads) {
                    const int h = hop[cur][i];
                    depth[cur ^ 1][i] = depth[cur][i] + depth[cur][h];
                    hop[cur ^ 1][i] = hop[cur][h];
                }
                __syncthreads();
                cur ^= 1;
            }
            const int L = p.seq_lens[b];
            bool far = L < 0;
            if (p.rope && !bad_tree)
                for (int i = tid; i < p.T; i += kThreads) far |= (int64_t)L + depth[cur][i] > p.max_positions;
            const bool no_room = __syncthreads_or(far);
            if (j == 0 && tid == 0) p.status[b] = bad_tree ? READER_ERR_BAD_TREE : no_room ? READER_ERR_CAPACITY : READER_OK;
            if (bad_tree || no_room) return 0;
            t.load_table(p, (int64_t)L + depth[cur][j] - 1);
            return 1;
        },
        [&](int x) -> uint4 * {
            if (x < p.Hq) return reinterpret_cast<uint4 *>(p.q_out + (row * p.Hq + x) * D);
            if (x < p.Hq + p.Hkv) return reinterpret_cast<uint4 *>(p.k_out + (row * p.Hkv + x - p.Hq) * D);
            return reinterpret_cast<uint4 *>(p.v_out + (row * p.Hkv + x - p.Hq - p.Hkv) * D);
        });
}

}  // namespace

void launch_prompt_append(const RotateParams &p, cudaStream_t st) {
    launch_pdl(p.D == 128 ? prompt_append_kernel<128> : prompt_append_kernel<64>, dim3((unsigned)(p.tokens + p.B)), dim3(kThreads), 0, st, p);
}

void launch_tree_rotate(const RotateParams &p, cudaStream_t st) {
    launch_pdl(p.D == 128 ? tree_rotate_kernel<128> : tree_rotate_kernel<64>, dim3((unsigned)(p.T * p.B)), dim3(kThreads), 0, st, p);
}

}  // namespace reader

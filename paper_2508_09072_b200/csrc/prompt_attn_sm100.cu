// Causal attention of packed prompts over the paged cache on the sm_100a tensor cores (reader_prompt_attn).
//
// Query i of a sequence stands at position L + i and sees the keys 0 .. L + i, all of them in the cache.  One CTA
// per SM walks its range of the unit list (prompt_attn.cuh).  It holds two 128-row query tiles and runs two
// independent softmax streams ("slots") beside each other, so that the tensor pipe works for one slot while the
// other slot's scores become probabilities:
//
//   warps 0-3, 4-7  softmax of slot 0 / 1: thread = query row, so a row's maximum and sum need no exchange
//   warp 8          producer: K and V tiles of 128 keys (two cache pages) by TMA through one ring, in the order in
//                   which they are multiplied; the query tiles of the next segment
//   warps 9, 11     issue S = Q K^T and O += P V of slot 0 / 1
//   warp 10         prepares the value tiles that hold keys some query of the unit does not see
//
// TMEM (512 columns): scores of slot 0 and 1 (128 columns each, fp32), outputs of slot 0 and 1 (D columns each).  The
// probabilities (bf16 pairs, 64 columns) take the place of their scores.  S(i+1) of a slot is issued behind PV(i),
// which reads P(i) from the same columns, and the tensor pipe runs the products that a thread issues in their order.
// P comes in two halves of 64 keys, so that the first half's product runs beside the second half's exponentials.
//
// Softmax: the exponentials of a tile are taken against the maximum known from the tiles before it while the tile's
// own maximum is found on the side; only if that exceeds the old one by more than 2^8 is the maximum raised, the
// output rescaled and the half done again (a segment's first tile looks for its maximum first).  Scores whose rounding
// exceeds what an exponential can hold (2^29 and up) take a slower path, tile by tile.  Scores, maxima, sums and
// outputs are fp32; P is rounded to bf16 for the value product (relative error of a weight 2^-8 at most, of the size
// of the output's own rounding), the row sum adds the unrounded weights.
//
// Keys that a row does not see get the score -inf by selection, whatever the cache holds there.  Values cannot be
// selected in a matrix product (0 * inf is NaN), so warp 10 goes over the tiles that hold keys of the unit's own
// tokens: rows behind the unit's last key are not multiplied or zeroed; an infinity or NaN in a row that some of the
// queries see is replaced by zero, and the epilogue adds it to exactly the rows that see it.
//
// Output rows leave through shared memory, 4 KB a warp: a warp's store then fills whole 128-byte lines.  (Straight from the
// thread = row layout, 16 bytes of 32 lines at a time, a segment's epilogue took 5500 to 9400 cycles.)
//
// A call with no more units than CTAs, all of them short, is this one launch (the single-launch form): a unit's CTA looks
// at its sequence's pages itself, writes zero rows if one is bad, and the status word if the unit is the sequence's first.
// Other calls are followed by the finishing kernel below.
//
// Every wait is bounded: a CTA that waits a second without progress marks its word in the workspace, stops waiting
// and runs to its end; the finishing kernel turns the mark into status words and zero rows.  In the single-launch form the
// CTA itself zeroes its unit's rows and sees to the status word (note_late).
#include <cuda.h>

#include "prompt_attn.cuh"
#include "prompt_ptx.cuh"

namespace reader {
namespace {

using namespace ptx;

constexpr int kThreads = 12 * 32;   // three warpgroups: two of softmax, one of single warps
// 168 registers a thread at launch; the softmax warpgroups take what the third can spare: 2 * 208 + 88 = 3 * 168
constexpr int kRegsSoftmax = 208, kRegsOther = 88;
constexpr int kProducerWarp = 8, kMmaWarp = 9, kValueWarp = 10;
constexpr uint64_t kWaitLimitNs = 1000000000ull;
constexpr float kRaiseMaxBy = 8.f;   // log2 units
constexpr float kHugeScore = 536870912.f;
// -infinity: every tile takes the slow path
__device__ __forceinline__ float margin_of(float mx) { return fabsf(mx) > kHugeScore && fabsf(mx) < INFINITY ? -INFINITY : kRaiseMaxBy; }
constexpr uint32_t kTmemCols = 512, kTmemS = 0, kTmemO = 256;
constexpr int kMaxStages = 8;
// Lengths of pieces, in key tiles, from which a form is taken.  Measured, us at 32/8/128 heads:
//   slot 1 begins half a step late, from 6, from 20, never: four prompts of 6001 to 8192 1600, 1599, 1608; two pieces on 30 k
//     histories 972, 932, 962; 16 prompts of up to 2048 313, 304, 304; a prompt of 4096 155, 153, 153
//   begun in the middle, from 16, from 64, never: the two pieces 928, 921, 957; 6 x 300 tokens on 2000 to 4000 133, 130, 130
//   values looked at ahead of their tiles, always, from 12, never: 5 prompts of 33 to 700 (8/8/64) 27.6, 20.6, 20.6; the 16
//     prompts 315, 304, 303; the prompt of 4096 154, 149, 155; the two pieces 936, 950, 953
constexpr int kLateStartTiles = 20, kRotateTiles = 64, kLookAheadTiles = 12;
constexpr int kMiscBytes = 3072;

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;                   // 64-column (128-byte) blocks per row
    static constexpr int kBlockBytes = 128 * 128;            // one 64-column block of 128 rows
    static constexpr int kTileBytes = kHalves * kBlockBytes; // a query, key or value tile
    static constexpr int kStages = D == 128 ? 4 : 8;
    static constexpr int kOffRing = 2 * kTileBytes;
    static constexpr int kOffStaging = kOffRing + kStages * kTileBytes;   // 4 KB per softmax warp
    static constexpr int kOffMisc = kOffStaging + 8 * 4096;
    static constexpr int kSmemBytes = kOffMisc + kMiscBytes;
};

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int32_t *abort_s) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_s) return false;
    const uint64_t t0 = globaltimer_ns();
    while (true) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*abort_s) return false;
        if (globaltimer_ns() - t0 > kWaitLimitNs) {
            *abort_s = 1;
            return false;
        }
    }
}

// A CTA's piece of a unit.
struct Piece {
    int b, h, block;
    int start;               // first row of the sequence in the packed tensors
    int L, n;
    UnitShape u;
    int t0, nt, rot;         // key tiles of this piece: t0 + (rot + j) % nt, j = 0 .. nt-1; nt = 0: no more work
    bool full;               // the whole unit
    int slot;                // where its partial goes
    int first_token;         // of the unit, within the sequence
    int32_t poison;          // infinities or NaN were taken out of its value tiles
    bool once;               // nobody else reads the keys and values of this piece
    bool reject;             // (single-launch form) a page id of the sequence is outside the pool: zero rows
    __device__ __forceinline__ int tile(int j) const { return t0 + (j + rot < nt ? j + rot : j + rot - nt); }
};

constexpr int kPieces = 4;          // pieces in flight between the producer and the other warps
constexpr int kConsumers = 11;      // those

struct Misc {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t raw[kMaxStages];  // a value tile that the value warp goes over first has landed; that warp then completes `full`
    uint64_t q_full, q_empty, s_full[2], p_full[2][2], o_full[2], turn[2], merge_ready, merge_free;
    uint64_t piece_full[kPieces], piece_empty[kPieces];
    float2 ml[128];            // slot 1's row maxima and sums of a narrow unit
    Piece piece[kPieces];
    uint32_t tmem_base;
    int32_t abort;
};
static_assert(sizeof(Misc) <= kMiscBytes, "shared memory behind the staging");

__device__ __forceinline__ int inclusive_sum(int x, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += up;
    }
    return x;
}

// Where a CTA's work comes from; one warp (the producer) asks, all its lanes together.
//   static (few units): the CTA's equal range of the unit list.  Pieces of a unit that is cut take its steps from the last
//     to the first, and a long unit is begun at the tile that the CTA's clock points to: CTAs that work on the same KV
//     head then ask for the same key tiles at about the same time, whatever part of the list they have, and a history
//     larger than the L2 cache is not fetched from HBM by each of them (2 x 32768 cached tokens: 2.95 GB without).
//   dynamic (many units): whole units from a counter, in the order (sequence, block from the last to the first, KV head):
//     the longest come first, the heads of one or two sequences fit the L2 cache.
//   alone (no more units than CTAs, all of them short): CTA i has unit i and nothing follows the kernel, see below.
struct Schedule {
    int w, left, w0, W, ctas;                    // static: place in the list, entries to go, where the range began
    int b, h, block, off, start, L, n, blocks;   // the current sequence, and the place in its unit
    int first;                                   // dynamic: units before sequence b

    __device__ __forceinline__ int blocks_of(const PromptAttnParams &p, int seq, int &n_, int &L_) const {
        n_ = p.token_start[seq + 1] - p.token_start[seq];
        L_ = p.seq_lens[seq];
        return prompt_len_ok(L_, n_, p.max_pages) ? unit_blocks(n_, p.tile_tokens) : 0;
    }
    __device__ __forceinline__ void open(const PromptAttnParams &p) {
        start = p.token_start[b];
        blocks = blocks_of(p, b, n, L);
    }
    // The single-launch form's only piece: unit blockIdx.x.  One look at the lengths, 32 sequences at a time.
    __device__ __forceinline__ bool alone(const PromptAttnParams &p, Piece &s, int lane) {
        const int i = blockIdx.x;
        bool bad = false, found = false;
        first = b = h = block = start = L = n = blocks = 0;
        s.nt = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            int a = 0, n_ = 0, L_ = 0, m = 0;
            if (b0 + lane < p.B) {
                a = p.token_start[b0 + lane];
                const int e = p.token_start[b0 + lane + 1];
                L_ = p.seq_lens[b0 + lane];
                bad |= a < 0 || a > e || e > p.tokens;
                n_ = e - a;
                if (!bad && prompt_len_ok(L_, n_, p.max_pages)) m = unit_blocks(n_, p.tile_tokens);
            }
            const int incl = inclusive_sum(m * p.Hkv, lane);
            const unsigned here = __ballot_sync(0xffffffffu, i - first < incl);
            if (here && !found) {
                const int src = __ffs(here) - 1;
                found = true;
                b = b0 + src;
                start = __shfl_sync(0xffffffffu, a, src);
                n = __shfl_sync(0xffffffffu, n_, src);
                L = __shfl_sync(0xffffffffu, L_, src);
                blocks = __shfl_sync(0xffffffffu, m, src);
                block = i - first - __shfl_sync(0xffffffffu, incl - m * p.Hkv, src);   // its place among the sequence's units
            }
            first += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (__any_sync(0xffffffffu, bad) || !found) return false;
        h = block % p.Hkv;
        block = block / p.Hkv;
        describe(p, s);
        s.t0 = 0;
        s.nt = s.u.tiles;
        s.full = true;
        s.slot = 0;
        return true;
    }
    // sizes: scratch in shared memory, [B]
    __device__ __forceinline__ void init(const PromptAttnParams &p, int32_t *sizes, int lane) {
        w = left = w0 = W = ctas = b = h = block = off = start = L = n = blocks = first = 0;
        const bool dealt = !p.counter;
        bool bad = false;
        int total = 0;   // entries of one head of every sequence so far
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            int n_ = 0, L_ = 0, m = 0, sum = 0;
            if (b0 + lane < p.B) {
                const int a = p.token_start[b0 + lane], e = p.token_start[b0 + lane + 1];
                L_ = p.seq_lens[b0 + lane];
                bad |= a < 0 || a > e || e > p.tokens;
                n_ = e - a;
                if (dealt && !bad && prompt_len_ok(L_, n_, p.max_pages)) m = unit_blocks(n_, p.tile_tokens);
            }
            if (!dealt) continue;
            // few blocks: each lane adds up its own sequence; many: the warp one sequence after the other
            for (int i = 0; m <= 4 && i < m; ++i) sum += unit_shape(L_, n_, i, p.tile_tokens).entries();
            for (unsigned long_ones = __ballot_sync(0xffffffffu, m > 4); long_ones; long_ones &= long_ones - 1) {
                const int src = __ffs(long_ones) - 1;
                const int ns = __shfl_sync(0xffffffffu, n_, src), Ls = __shfl_sync(0xffffffffu, L_, src), ms = __shfl_sync(0xffffffffu, m, src);
                int part = 0;
                for (int i = lane; i < ms; i += 32) part += unit_shape(Ls, ns, i, p.tile_tokens).entries();
                part = __reduce_add_sync(0xffffffffu, part);
                if (lane == src) sum = part;
            }
            const int incl = inclusive_sum(sum, lane);
            if (b0 + lane < p.B) sizes[b0 + lane] = total + incl - sum;
            total += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (__any_sync(0xffffffffu, bad)) {   // whose rows are whose is not known: no work
            b = p.B;
            return;
        }
        if (!dealt) return;
        __syncwarp();
        W = total * p.Hkv;
        ctas = prompt_busy_ctas(p.n_ctas, W);
        const int c = blockIdx.x;
        if (c >= ctas) return;
        w0 = w = prompt_range_begin(c, W, ctas);
        left = prompt_range_begin(c + 1, W, ctas) - w;
        if (left <= 0) return;
        int lo = 0, hi = p.B;   // the last sequence that begins at or before this CTA's first entry
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (sizes[mid] * p.Hkv <= w) lo = mid; else hi = mid;
        }
        b = lo;
        const int size = (b + 1 < p.B ? sizes[b + 1] : total) - sizes[b], within = w - sizes[b] * p.Hkv;
        h = within / size;
        off = within - h * size;
        open(p);
        for (int i0 = 0; i0 < blocks; i0 += 32) {
            const int mine = i0 + lane < blocks ? unit_shape(L, n, i0 + lane, p.tile_tokens).entries() : 0;
            const int incl = inclusive_sum(mine, lane);
            const unsigned here = __ballot_sync(0xffffffffu, off < incl);
            if (here) {
                const int src = __ffs(here) - 1;
                block = i0 + src;
                off -= __shfl_sync(0xffffffffu, incl - mine, src);
                break;
            }
            off -= __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    __device__ __forceinline__ void describe(const PromptAttnParams &p, Piece &s) const {
        s.b = b; s.h = h; s.block = block;
        s.start = start; s.L = L; s.n = n;
        s.u = unit_shape(L, n, block, p.tile_tokens);
        s.first_token = block * 2 * p.tile_tokens;
        s.rot = 0;
        s.poison = 0;
        s.once = blocks == 1 && p.shared_prefix_len == 0;
        s.reject = false;
    }
    // The next piece with at least one key tile; false when there is no more.
    __device__ __forceinline__ bool next(const PromptAttnParams &p, Piece &s, int lane) {
        s.nt = 0;
        if (p.counter) {
            if (b >= p.B) return false;
            int i = 0;
            if (lane == 0) i = atomicAdd(p.counter, 1);
            i = __shfl_sync(0xffffffffu, i, 0);
            while (true) {
                int n_ = 0, L_ = 0, m = 0;
                if (b + lane < p.B) m = blocks_of(p, b + lane, n_, L_) * p.Hkv;
                const int incl = inclusive_sum(m, lane);
                const unsigned here = __ballot_sync(0xffffffffu, i - first < incl);
                if (here) {
                    const int src = __ffs(here) - 1;
                    b += src;
                    first += __shfl_sync(0xffffffffu, incl - m, src);
                    break;
                }
                b += 32;
                first += __shfl_sync(0xffffffffu, incl, 31);
                if (b >= p.B) return false;
            }
            open(p);
            block = blocks - 1 - (i - first) / p.Hkv;
            h = (i - first) % p.Hkv;
            describe(p, s);
            s.t0 = 0;
            s.nt = s.u.tiles;
            s.full = true;
            s.slot = 0;
            return true;
        }
        while (left > 0) {
            while (block >= blocks) {   // on to the next head, the next sequence with tokens
                block = 0;
                if (blocks == 0 || ++h == p.Hkv) {
                    h = 0;
                    if (++b >= p.B) {
                        left = 0;
                        return false;
                    }
                    open(p);
                }
            }
            describe(p, s);
            const int entries = s.u.entries(), extra = entries - s.u.steps, take = min(entries - off, left);
            const int s0 = max(0, off - extra), s1 = off + take - extra;
            const int per = s.u.narrow ? 2 : 1;   // tiles a step
            if (s1 > s0) {
                s.t0 = max(0, s.u.tiles - per * s1);
                s.nt = s.u.tiles - per * s0 - s.t0;
            }
            s.full = s0 == 0 && s1 == s.u.steps;
            s.slot = s0 == 0 ? 1 : 0;
            if (s.full && s.nt >= kRotateTiles) s.rot = per * (w - w0) % s.nt;
            w += take;
            left -= take;
            off += take;
            const int rest = s.u.steps - s1;   // of the unit, with the CTAs that follow
            if (s.nt > 0 && !s.full && s.slot == 1 && lane == 0) {
                PieceDesc d;
                d.b = b; d.h = h; d.block = block;
                d.more = prompt_range_owner(w + rest - 1, W, ctas) - (int)blockIdx.x;
                d.first_token = start; d.tokens = n; d.L = L;
                p.pieces[blockIdx.x] = d;
            }
            if (off == entries) { off = 0; ++block; }
            if (s.nt > 0) return true;
        }
        return false;
    }
};

// Ring places of a segment's tiles.  Order: the first `ahead` key tiles, then V0, K(ahead), V1, K(ahead + 1), ...
__device__ __forceinline__ int ahead_of(const Piece &s) { return min(s.u.narrow ? 2 : 1, s.nt); }
__device__ __forceinline__ int place_of_k(int j, int ahead) { return j < ahead ? j : ahead + 2 * (j - ahead) + 1; }
__device__ __forceinline__ int place_of_v(int j, int ahead, int nt) { return ahead + j + min(j, nt - ahead); }

// Whether key tile t holds keys of the unit's own tokens (or none): its values go through the value warp.
__device__ __forceinline__ bool has_own_keys(const Piece &s, int t) { return (t + 1) * kKeyTile > s.L + s.first_token; }

// Page ids of a piece's key tiles, 16 tiles at a time (one id per lane).
struct PageCursor {
    int t_first = 0, id = 0;
    bool loaded = false;
    __device__ __forceinline__ void get(const PromptAttnParams &p, const Piece &s, int t, int lane, int &a, int &b) {
        if (!loaded || (unsigned)(t - t_first) >= 16u) {
            t_first = t;
            const int i = 2 * t + lane, npages = (s.u.keys + kPage - 1) / kPage;
            id = i < npages ? p.page_table[(size_t)s.b * p.max_pages + i] : 0;
            loaded = true;
        }
        a = __shfl_sync(0xffffffffu, id, 2 * (t - t_first));
        b = __shfl_sync(0xffffffffu, id, 2 * (t - t_first) + 1);
    }
};

__device__ __forceinline__ void zero_sequence(const PromptAttnParams &p, int b, int D, int t, int threads) {
    const int start = p.token_start[b], n = p.token_start[b + 1] - start;
    uint4 *rows = reinterpret_cast<uint4 *>(p.out + (size_t)start * p.Hq * D);
    for (size_t i = t; i < (size_t)n * p.Hq * D / 8; i += threads) rows[i] = make_uint4(0, 0, 0, 0);
    if (p.lse)
        for (size_t i = t; i < (size_t)n * p.Hq; i += threads) p.lse[(size_t)start * p.Hq + i] = 0.f;
}

// Single-launch form: the status words of the sequences without a unit, and zero rows for those of them that have rows.
// (A sequence with units is reported by the CTA of its first one.)  One warp of one CTA.
template <int D>
__device__ void report_idle(const PromptAttnParams &p, int lane) {
    bool bad = false;
    for (int b = lane; b < p.B; b += 32) {
        const int a = p.token_start[b], e = p.token_start[b + 1];
        bad |= a < 0 || a > e || e > p.tokens;
    }
    const bool none = __any_sync(0xffffffffu, bad);
    for (int b0 = 0; b0 < p.B; b0 += 32) {
        const int b = b0 + lane;
        bool wrong = false;
        if (b < p.B) {
            const int n = p.token_start[b + 1] - p.token_start[b];
            wrong = !none && !prompt_len_ok(p.seq_lens[b], n, p.max_pages);
            if (none || wrong || n == 0) p.status[b] = none ? READER_ERR_INVALID_ARG : wrong ? READER_ERR_CAPACITY : READER_OK;
        }
        for (unsigned left = __ballot_sync(0xffffffffu, wrong); left; left &= left - 1) zero_sequence(p, b0 + __ffs(left) - 1, D, lane, 32);
    }
}

// Single-launch form: the status word of a sequence whose units several CTAs do.  The CTA of its first unit (`first`) writes it
// (report), and one that gives up, READER_ERR_TIMEOUT (note_late), in no order: the first unit's CTA may even start after
// another one's second has passed.  So that the error is what stays, the one that gives up leaves a note before it writes,
// and the other one looks for the note after it has written: whichever write is the last, it is the error.  (A note may come
// after that look, and is then found by the next call that puts the sequence's units on the same CTA with the same
// workspace: a call that gave up can be reported once more, never less.)
__device__ __forceinline__ void note_late(const PromptAttnParams &p, int b, int first) {
    *(volatile uint64_t *)&p.late_notes[first] = kLateNote;
    __threadfence();
    *(volatile int32_t *)&p.status[b] = READER_ERR_TIMEOUT;
}
__device__ __forceinline__ void report(const PromptAttnParams &p, int b, int first, int status) {
    *(volatile int32_t *)&p.status[b] = status;
    __threadfence();
    if (*(volatile uint64_t *)&p.late_notes[first] == kLateNote) {
        *(volatile uint64_t *)&p.late_notes[first] = 0;
        *(volatile int32_t *)&p.status[b] = READER_ERR_TIMEOUT;
    }
}

__device__ __forceinline__ bool nonfinite_bits(uint32_t half) { return (half & 0x7f80u) == 0x7f80u; }

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
prompt_attn_kernel(const PromptAttnParams p, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                   const __grid_constant__ CUtensorMap vmap, const __nv_bfloat16 *v_pool) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (base & 1023u) {   // the swizzled tiles need 1024-byte alignment; never seen, but checked (it is the same for all CTAs)
        grid_dependency_wait();
        if (tid == 0) {
            p.gave_up[blockIdx.x] = 1;
            p.pieces[blockIdx.x].b = -1;
        }
        for (int b = tid; p.alone && blockIdx.x == 0 && b < p.B; b += kThreads) p.status[b] = READER_ERR_CUDA;
        return;
    }
    Misc *m = reinterpret_cast<Misc *>(smem + C::kOffMisc);
    volatile int32_t *abort_s = &m->abort;
    const uint32_t sQ = base, sRing = base + C::kOffRing;
    auto bar = [&](const uint64_t *b) { return smem_u32(b); };

    if (tid == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(bar(&m->full[i]), 1);
            mbar_init(bar(&m->empty[i]), 2);   // both slots
            mbar_init(bar(&m->raw[i]), 1);
        }
        mbar_init(bar(&m->q_full), 1);
        mbar_init(bar(&m->q_empty), 2);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(&m->s_full[s]), 1);
            mbar_init(bar(&m->p_full[s][0]), 128);
            mbar_init(bar(&m->p_full[s][1]), 128);
            mbar_init(bar(&m->o_full[s]), 1);
            mbar_init(bar(&m->turn[s]), 1);
        }
        mbar_init(bar(&m->merge_ready), 128);
        mbar_init(bar(&m->merge_free), 128);
        m->abort = 0;
        m->piece[0].nt = 0;
        for (int i = 0; i < kPieces; ++i) {
            mbar_init(bar(&m->piece_full[i]), 1);
            mbar_init(bar(&m->piece_empty[i]), kConsumers);
        }
        fence_mbar_init();
        mbar_arrive(bar(&m->turn[0]));   // slot 0 has the first turn
        fence_proxy_async();
        prefetch_tensormap(&qmap);
        prefetch_tensormap(&kmap);
        prefetch_tensormap(&vmap);
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&m->tmem_base), kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = m->tmem_base;
    // everything above overlapped the kernel before this one in the stream; its results are read from here on
    grid_dependency_wait();
    grid_launch_dependents();
    // the piece a warp is working on
    int pieces = 0;
    const Piece *sg = m->piece;
    auto next = [&]() -> bool {
        const int i = pieces % kPieces;
        if (!wait(bar(&m->piece_full[i]), (pieces / kPieces) & 1, abort_s)) return false;
        ++pieces;
        sg = &m->piece[i];
        return sg->nt > 0;
    };
    auto done = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(&m->piece_empty[(pieces - 1) % kPieces]));
    };
    if (warp >= 8) {
        regs_dec<kRegsOther>();
        if (warp == kProducerWarp) {
            // ------------------------------------------------------------------ producer
            int r = 0, seg = 0;
            if (lane == 0) p.pieces[blockIdx.x].b = -1;
            __syncwarp();
            Schedule schedule;
            if (!p.alone) {
                schedule.init(p, reinterpret_cast<int32_t *>(smem + C::kOffRing), lane);
                // the ring was every lane's scratch until here: each orders its own accesses before the copies that one of them issues
                fence_proxy_async();
                __syncwarp();
            }
            Piece s;
            const uint64_t stream_policy = l2_policy_evict_first();
            auto load = [&](PageCursor &cursor, const CUtensorMap *map, int j, bool values) {
                const int stage = r % C::kStages, t = s.tile(j), npg = t * kKeyTile + kPage < s.u.keys ? 2 : 1;
                int page_a, page_b;
                cursor.get(p, s, t, lane, page_a, page_b);
                const bool ok = wait(bar(&m->empty[stage]), ((r / C::kStages) & 1) ^ 1, abort_s);
                __syncwarp();
                if (ok && elect_one()) {
                    const uint32_t full = bar(values && has_own_keys(s, t) ? &m->raw[stage] : &m->full[stage]), dst = sRing + stage * C::kTileBytes;
                    mbar_arrive_expect_tx(full, npg * (C::kTileBytes / 2));
                    const int row_a = (page_a * p.Hkv + s.h) * kPage, row_b = (page_b * p.Hkv + s.h) * kPage;
#pragma unroll
                    for (int hf = 0; hf < C::kHalves; ++hf) {
                        // what is read once should not push lines that others will ask for out of L2
                        const uint32_t to = dst + hf * C::kBlockBytes;
                        if (s.once) tma_load_2d_hint(to, map, full, hf * 64, row_a, stream_policy);
                        else tma_load_2d(to, map, full, hf * 64, row_a);
                        if (npg > 1 && s.once) tma_load_2d_hint(to + C::kBlockBytes / 2, map, full, hf * 64, row_b, stream_policy);
                        else if (npg > 1) tma_load_2d(to + C::kBlockBytes / 2, map, full, hf * 64, row_b);
                    }
                }
                __syncwarp();
                ++r;
            };
            const int tile_rows_bytes = p.G * p.tile_tokens * 128;
            while (!*abort_s) {
                bool more;
                if (!p.alone) more = schedule.next(p, s, lane);
                else if (seg == 0) more = schedule.alone(p, s, lane);
                else more = false;
                if (!more) s.nt = 0;
                const int i = seg % kPieces;
                if (!wait(bar(&m->piece_empty[i]), ((seg / kPieces) & 1) ^ 1, abort_s)) break;
                if (lane == 0) {
                    m->piece[i] = s;
                    mbar_arrive(bar(&m->piece_full[i]));
                }
                __syncwarp();
                if (!more) break;
                const int ahead = ahead_of(s);
                PageCursor kc, vc;
                bool bad_page = false;
                if (p.alone) {   // the sequence's pages, to be looked at below; the first 32 serve the loads too
                    const int npages = (s.L + s.n + kPage - 1) / kPage;
                    kc.loaded = vc.loaded = true;
                    if (lane < npages) {
                        kc.id = p.page_table[(size_t)s.b * p.max_pages + lane];
                        bad_page = kc.id < 0 || kc.id >= p.num_pages;
                    }
                    vc.id = kc.id;
                }
                for (int j = 0; j < ahead; ++j) load(kc, &kmap, j, false);
                if (wait(bar(&m->q_empty), (seg & 1) ^ 1, abort_s) && elect_one()) {
                    const uint32_t full = bar(&m->q_full);
                    const int tiles = s.u.narrow ? 1 : 2;
                    mbar_arrive_expect_tx(full, tiles * C::kHalves * tile_rows_bytes);
                    for (int q = 0; q < tiles; ++q)
#pragma unroll
                        for (int hf = 0; hf < C::kHalves; ++hf)
                            tma_load_3d(sQ + q * C::kTileBytes + hf * C::kBlockBytes, &qmap, full, hf * 64, s.h * p.G,
                                        s.start + s.first_token + q * p.tile_tokens);
                }
                __syncwarp();
                ++seg;
                if (p.alone) {
                    for (int k = 32 + lane; k < (s.L + s.n + kPage - 1) / kPage; k += 32) {
                        const int pg = p.page_table[(size_t)s.b * p.max_pages + k];
                        bad_page |= pg < 0 || pg >= p.num_pages;
                    }
                    const bool reject = __any_sync(0xffffffffu, bad_page);
                    if (reject && lane == 0) *(volatile bool *)&m->piece[i].reject = true;   // (before the values are asked for)
                    __syncwarp();
                }
                for (int j = 0; j < s.nt; ++j) {
                    load(vc, &vmap, j, true);
                    if (j + ahead < s.nt) load(kc, &kmap, j + ahead, false);
                }
                // (beside the last products and the epilogue this takes no time)
                if (p.alone && s.h == 0 && s.block == 0 && lane == 0) report(p, s.b, blockIdx.x, m->piece[0].reject ? READER_ERR_BAD_PAGE : READER_OK);
                __syncwarp();
            }
            // a CTA that gave up must not exit under its own copies: let the last ones land (bounded)
            if (*abort_s) {
                const uint64_t t0 = globaltimer_ns();
                for (int i = max(0, r - C::kStages); i < r; ++i)
                    while (!mbar_try_wait(bar(&m->full[i % C::kStages]), (i / C::kStages) & 1) && globaltimer_ns() - t0 < 20000000ull) {
                    }
                if (seg > 0)
                    while (!mbar_try_wait(bar(&m->q_full), (seg - 1) & 1) && globaltimer_ns() - t0 < 20000000ull) {
                    }
            }
        } else if (warp != kValueWarp) {
            // ------------------------------------------------------------------ issuer of a slot's products
            const int slot = warp == kMmaWarp ? 0 : 1;
            constexpr uint32_t kIdescQK = idesc_bf16_f32(128, kKeyTile, false, false);
            constexpr uint32_t kIdescPV = idesc_bf16_f32(128, D, false, true);
            const uint64_t descQ = smem_desc_sw128(sQ, 16, 1024), descK = smem_desc_sw128(sRing, 16, 1024);
            const uint64_t descV = smem_desc_sw128(sRing, C::kBlockBytes, 1024);
            const uint32_t tS = tmem + kTmemS + slot * 128, tO = tmem + kTmemO + slot * D;
            int r = 0, seg = 0;   // r: the next place in the ring that this warp has not seen
            uint32_t p_parity = 0, turn_parity = 0;
            auto wait_full = [&](int place) { wait(bar(&m->full[place % C::kStages]), (place / C::kStages) & 1, abort_s); };
            // Both issuers see every tile in the ring's order, so that neither can fall a whole turn behind (a parity wait
            // tells a phase only from the one before it); tiles of the other slot are passed on at once.
            auto pass_to = [&](int place) {
                for (; r < place; ++r) {
                    wait_full(r);
                    if (lane == 0) mbar_arrive(bar(&m->empty[r % C::kStages]));
                }
                __syncwarp();
            };
            auto issue_s = [&](uint64_t qd, int place, bool last) {
                const uint64_t kd = descK + (uint64_t)(((place % C::kStages) * C::kTileBytes) >> 4);
#pragma unroll
                for (int hf = 0; hf < C::kHalves; ++hf)
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_bf16_ss(tS, qd + (uint64_t)((hf * C::kBlockBytes + kk * 32) >> 4),
                                    kd + (uint64_t)((hf * C::kBlockBytes + kk * 32) >> 4), kIdescQK, (hf | kk) != 0);
                mma_commit(bar(&m->s_full[slot]));
                mma_commit(bar(&m->empty[place % C::kStages]));
                if (last) mma_commit(bar(&m->q_empty));
            };
            // half 0: the first 64 keys of the tile, half 1: the others
            auto issue_pv = [&](int half, int place, int slices, bool first) {
                const uint64_t vd = descV + (uint64_t)(((place % C::kStages) * C::kTileBytes) >> 4);
#pragma unroll
                for (int k4 = 0; k4 < 4; ++k4) {
                    const int kk = half * 4 + k4;
                    if (kk < slices) mma_bf16_ts(tO, tS + kk * 8, vd + (uint64_t)((kk * 2048) >> 4), kIdescPV, !first || kk != 0);
                }
            };
            while (!*abort_s && next()) {
                const int ahead = ahead_of(*sg), n = sg->nt, r0 = r, keys = sg->u.keys;
                const bool narrow = sg->u.narrow;
                const int j0 = narrow ? slot : 0, dj = narrow ? 2 : 1;
                const uint64_t qd = descQ + (uint64_t)((narrow ? 0 : slot * C::kTileBytes) >> 4);
                // Left to themselves the two slots fall into step, score products side by side and then both softmaxes
                // on the special-function units at once (3970 cycles a step).  In a wide unit they therefore take turns with
                // their score products, slot 0 first: each slot's softmax then runs beside the other's products.
                // How far slot 1 begins behind slot 0 is how far it stays: in a long piece it waits for slot 0's first
                // probabilities, half a step (attn_long 1630 -> 1586 us; in a short piece the wait costs more than it brings).
                const bool late_start = !narrow && slot == 0 && n >= kLateStartTiles;
                auto take_turn = [&]() {
                    if (!narrow) wait(bar(&m->turn[slot]), turn_parity, abort_s);
                    turn_parity ^= narrow ? 0 : 1;
                };
                auto pass_turn = [&]() {
                    if (!narrow && lane == 0) mbar_arrive(bar(&m->turn[slot ^ 1]));
                    __syncwarp();
                };
                wait(bar(&m->q_full), seg & 1, abort_s);
                ++seg;
                if (j0 < n) {
                    pass_to(r0 + place_of_k(j0, ahead));
                    wait_full(r);
                    take_turn();
                    tc_fence_after();
                    __syncwarp();
                    if (elect_one()) issue_s(qd, r, j0 + dj >= n);
                    __syncwarp();
                    if (!late_start) pass_turn();
                    ++r;
                    for (int j = j0; j < n; j += dj) {
                        const int slices = (min(kKeyTile, keys - sg->tile(j) * kKeyTile) + 15) >> 4;
                        const bool more = j + dj < n;
                        pass_to(r0 + place_of_v(j, ahead, n));
                        const int rv = r;
                        wait_full(r++);
                        wait(bar(&m->p_full[slot][0]), p_parity, abort_s);
                        tc_fence_after();
                        __syncwarp();
                        if (elect_one()) issue_pv(0, rv, slices, j == j0);
                        __syncwarp();
                        if (late_start && j == j0) pass_turn();
                        if (more) {
                            pass_to(r0 + place_of_k(j + dj, ahead));
                            wait_full(r);
                            take_turn();
                        }
                        wait(bar(&m->p_full[slot][1]), p_parity, abort_s);
                        p_parity ^= 1;
                        tc_fence_after();
                        __syncwarp();
                        if (elect_one()) {
                            issue_pv(1, rv, slices, j == j0);
                            mma_commit(bar(&m->empty[rv % C::kStages]));
                            if (more) issue_s(qd, r, j + 2 * dj >= n);
                            else mma_commit(bar(&m->o_full[slot]));
                        }
                        __syncwarp();
                        if (more) {
                            pass_turn();
                            ++r;
                        }
                    }
                } else {
                    if (lane == 0) mbar_arrive(bar(&m->q_empty));   // a narrow piece of one tile: slot 1 has none
                    __syncwarp();
                }
                pass_to(r0 + 2 * n);
                done();
            }
            if (*abort_s) __nanosleep(1000000);   // products that are still under way end before their operands go away
        } else if (warp == kValueWarp) {
            // ------------------------------------------------------------------ values some queries do not see; the note on a split unit
            int r0 = 0;
            uint32_t raw_parity = 0;   // one bit per ring stage
            if (p.alone && blockIdx.x == 0) report_idle<D>(p, lane);
            while (!*abort_s && next()) {
                const int ahead = ahead_of(*sg), n = sg->nt, own_key = sg->L + sg->first_token;
                constexpr int kChunks = D / 8;   // 16-byte pieces per row
                // A look at the exponents (all ones: infinity or NaN) of the value rows that are multiplied although some query does
                // not see them: the unit's own tokens, and what the last slice of 16 rows holds behind them.  They are read from
                // the pool, while the tiles are on their way: out of shared memory, whose bandwidth the products take up,
                // one tile took 6000 cycles.  (Plain loads: the kernel before may still have been writing these rows when this one was
                // launched, so they are not read-only for its lifetime.)
                const int lo = max(own_key, sg->t0 * kKeyTile), hi = min((sg->u.keys + 15) & ~15, (sg->t0 + n) * kKeyTile);
                // (A short piece has no time for that, and few products: its tiles are gone through in shared memory.)
                bool dirty = n < kLookAheadTiles;
                if (!dirty && lo < hi) {
                    constexpr int kBatch = 8;    // pieces a lane has in flight
                    const int first_page = lo / kPage;
                    int page = -1;
                    if (first_page + lane <= (hi - 1) / kPage) page = p.page_table[(size_t)sg->b * p.max_pages + first_page + lane];
                    if (page >= p.num_pages) page = -1;
                    uint32_t ones = 0;
                    for (int i0 = 0; i0 < (hi - lo) * kChunks; i0 += kBatch * 32) {
                        uint4 x[kBatch];
#pragma unroll
                        for (int k = 0; k < kBatch; ++k) {
                            const int i = i0 + k * 32 + lane, key = lo + i / kChunks;
                            const int pg = __shfl_sync(0xffffffffu, page, (key / kPage - first_page) & 31);
                            x[k] = make_uint4(0, 0, 0, 0);
                            if (key < hi && pg >= 0)
                                x[k] = *(reinterpret_cast<const uint4 *>(v_pool + (((size_t)pg * p.Hkv + sg->h) * kPage + key % kPage) * D) + i % kChunks);
                        }
#pragma unroll
                        for (int k = 0; k < kBatch; ++k) {
                            ones |= ((x[k].x & 0x7f807f80u) + 0x00800080u) | ((x[k].y & 0x7f807f80u) + 0x00800080u);
                            ones |= ((x[k].z & 0x7f807f80u) + 0x00800080u) | ((x[k].w & 0x7f807f80u) + 0x00800080u);
                        }
                    }
                    dirty = __any_sync(0xffffffffu, (ones & 0x80008000u) != 0);
                }
                for (int j = 0; j < n; ++j) {
                    const int t = sg->tile(j);
                    if (!has_own_keys(*sg, t)) continue;
                    const int r = r0 + place_of_v(j, ahead, n), stage = r % C::kStages;
                    if (!wait(bar(&m->raw[stage]), (raw_parity >> stage) & 1, abort_s)) break;
                    raw_parity ^= 1u << stage;
                    if (!dirty) {
                        if (lane == 0) mbar_arrive(bar(&m->full[stage]));
                        __syncwarp();
                        continue;
                    }
                    const uint32_t tile = sRing + stage * C::kTileBytes;
                    const int valid = min(kKeyTile, sg->u.keys - t * kKeyTile), end = (valid + 15) & ~15;
                    const int own_row = max(0, own_key - t * kKeyTile);
                    auto piece_at = [&](int i) {
                        const int row = i / kChunks, c = i % kChunks;
                        return tile + (c >> 3) * C::kBlockBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4);
                    };
                    bool found = false;
                    constexpr int kAtOnce = 8;
                    for (int i0 = own_row * kChunks + lane; i0 < valid * kChunks; i0 += kAtOnce * 32) {
                        uint32_t x[kAtOnce][4];
                        uint32_t ones = 0;
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            x[k][0] = x[k][1] = x[k][2] = x[k][3] = 0;
                            if (i0 + k * 32 < valid * kChunks)
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[k][0]), "=r"(x[k][1]), "=r"(x[k][2]), "=r"(x[k][3]) : "r"(piece_at(i0 + k * 32)));
                        }
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
                            for (int e = 0; e < 4; ++e) ones |= (x[k][e] & 0x7f807f80u) + 0x00800080u;
                        if (!(ones & 0x80008000u)) continue;
                        found = true;
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (nonfinite_bits(x[k][e])) x[k][e] &= 0xffff0000u;
                                if (nonfinite_bits(x[k][e] >> 16)) x[k][e] &= 0x0000ffffu;
                            }
                            if (i0 + k * 32 < valid * kChunks)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece_at(i0 + k * 32)), "r"(x[k][0]), "r"(x[k][1]), "r"(x[k][2]), "r"(x[k][3]) : "memory");
                        }
                    }
                    if (__any_sync(0xffffffffu, found) && lane == 0) *(volatile int32_t *)&m->piece[(pieces - 1) % kPieces].poison = 1;
                    for (int i = valid * kChunks + lane; i < end * kChunks; i += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(piece_at(i)), "r"(0u) : "memory");
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&m->full[stage]));
                }
                r0 += 2 * n;
                done();
            }
        }
    } else {
        // ------------------------------------------------------------------ softmax / epilogue
        regs_inc<kRegsSoftmax>();
        const int slot = warp >> 2, row = tid & 127;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + kTmemS + slot * 128 + lane_base, tO = tmem + kTmemO + slot * D + lane_base;
        constexpr uint32_t kNegInf = 0xff800000u;
        const int row_token = row / p.G, row_member = row - row_token * p.G;
        int narrows = 0;
        uint32_t s_parity = 0, o_parity = 0;
        while (next()) {
            const bool narrow = sg->u.narrow;
            const int unit_token = (narrow ? 0 : slot * p.tile_tokens) + row_token;   // within the unit
            const bool live = row_token < p.tile_tokens && unit_token < sg->u.tokens;
            const bool warp_live = __any_sync(0xffffffffu, live);
            // the last key this row sees; rows without a query see what the first row sees
            const int last_key = sg->L + sg->first_token + (live ? unit_token : 0);
            const int warp_min = __reduce_min_sync(0xffffffffu, last_key);
            // Running maximum (scaled, log2 units) and row sum.  A row without a query (it holds the next sequence's, or what an
            // earlier call left in shared memory) has the maximum +inf from the start: it never asks for a higher one, so the
            // rows that share its warp are computed as if it were not there.  (A margin of its own for such rows, or its vote
            // masked, costs a register in the loop: four long prompts 1600 us, this way 1578.)
            float mx = live ? -INFINITY : INFINITY, l = 0.f;
            const int j0 = narrow ? slot : 0, dj = narrow ? 2 : 1, nt = sg->nt;
            float margin = kRaiseMaxBy;       // the maximum is raised by scores that exceed it by more
            bool any = false;
            for (int j = j0; j < nt; j += dj) {
                const int key0 = sg->tile(j) * kKeyTile;
                wait(bar(&m->s_full[slot]), s_parity, abort_s);
                s_parity ^= 1;
                tc_fence_after();
                if (warp_live) {
                    uint32_t sc[128];
                    auto f = [&](int i) { return __uint_as_float(sc[i]); };
                    auto tile_top = [&]() {
                        float tops[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            float a = max3(f(c * 32), f(c * 32 + 1), f(c * 32 + 2));
#pragma unroll
                            for (int i = 3; i < 31; i += 2) a = max3(a, f(c * 32 + i), f(c * 32 + i + 1));
                            tops[c] = fmaxf(a, f(c * 32 + 31));
                        }
                        return fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]) * p.scale_log2;
                    };
                    const float2 sc2 = make_float2(p.scale_log2, p.scale_log2);
                    float2 neg2, part[2];
                    uint32_t pk[32];
                    auto exponentials = [&](int half) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const int at = half * 64 + 2 * i;
                            const float2 x = __ffma2_rn(make_float2(f(at), f(at + 1)), sc2, neg2);
                            const float2 e = make_float2(ex2(x.x), ex2(x.y));
                            part[i & 1] = __fadd2_rn(part[i & 1], e);
                            const __nv_bfloat162 hh = __floats2bfloat162_rn(e.x, e.y);
                            pk[i] = *reinterpret_cast<const uint32_t *>(&hh);
                        }
                    };
                    bool first = !any, huge = false;
                    while (true) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sc[c * 32]));
                        tmem_wait_ld();
                        if (key0 + kKeyTile - 1 > warp_min) {
                            const int lim = last_key - key0;   // columns 0 .. lim are seen
#pragma unroll
                            for (int i = 0; i < 128; ++i)
                                if (i > lim) sc[i] = kNegInf;
                        }
                        if (first) {
                            mx = fmaxf(mx, tile_top());   // (-inf where the row sees none of these keys)
                            margin = margin_of(mx);
                            first = false;
                        }
                        const float neg = mx == -INFINITY ? 0.f : -mx;
                        neg2 = make_float2(neg, neg);
                        part[0] = part[1] = make_float2(0.f, 0.f);
                        exponentials(0);
                        const float top = tile_top();
                        if (!__any_sync(0xffffffffu, top > mx + margin)) break;
                        const float up = fmaxf(mx, top);
                        const float alpha = up == -INFINITY ? 1.f : ex2(mx - up);
                        mx = up;
                        l *= alpha;
                        // (the scores of this tile are complete, hence the value product before them is)
#pragma unroll 1
                        for (int c = 0; any && c < D; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(tO + c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st16(tO + c, o);
                        }
                        margin = margin_of(mx);
                        if (__any_sync(0xffffffffu, margin != kRaiseMaxBy)) {
                            huge = true;
                            break;
                        }
                        tmem_wait_st();
                    }
                    if (__builtin_expect(huge, 0)) {
                        // Past 2^29 the rounding of the maximum is no longer small against what an exponential holds, and the
                        // fused product would keep it: here scores are scaled and rounded like the maximum before they meet.
                        const float neg = mx == -INFINITY ? 0.f : -mx;
#pragma unroll 1
                        for (int c = 0; c < kKeyTile; c += 32) {
                            uint32_t x[32];
                            tmem_ld32(tS + c, x);
                            tmem_wait_ld();
                            float e[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                e[i] = key0 + c + i > last_key ? 0.f : ex2(__fadd_rn(__fmul_rn(__uint_as_float(x[i]), p.scale_log2), neg));
                                l += e[i];
                            }
                            uint32_t y[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const __nv_bfloat162 hh = __floats2bfloat162_rn(e[2 * i], e[2 * i + 1]);
                                y[i] = *reinterpret_cast<const uint32_t *>(&hh);
                            }
                            tmem_st16(tS + c / 2, y);   // (columns that have been read)
                        }
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive(bar(&m->p_full[slot][0]));
                    } else {
                        tmem_st32(tS, pk);
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive(bar(&m->p_full[slot][0]));
                        exponentials(1);
                        tmem_st32(tS + 32, pk);
                        l += (part[0].x + part[1].x) + (part[0].y + part[1].y);
                        tmem_wait_st();
                    }
                } else {
                    tc_fence_before();
                    mbar_arrive(bar(&m->p_full[slot][0]));
                }
                any = true;
                tc_fence_before();
                mbar_arrive(bar(&m->p_full[slot][1]));
            }
            // ---- segment epilogue
            if (any) {
                wait(bar(&m->o_full[slot]), o_parity, abort_s);
                o_parity ^= 1;
                tc_fence_after();
            }
            float w0 = 1.f, w1 = 0.f, l_all = l, m_all = mx;
            if (narrow) {
                if (slot == 1) {
                    m->ml[row] = make_float2(mx, any ? l : 0.f);
                    tc_fence_before();
                    mbar_arrive(bar(&m->merge_ready));
                    wait(bar(&m->merge_free), narrows & 1, abort_s);
                    ++narrows;
                    done();
                    continue;
                }
                wait(bar(&m->merge_ready), narrows & 1, abort_s);
                tc_fence_after();
                const float2 other = m->ml[row];
                m_all = fmaxf(mx, other.x);
                w0 = mx == -INFINITY ? 0.f : ex2(mx - m_all);
                w1 = other.x == -INFINITY ? 0.f : ex2(other.x - m_all);
                l_all = l * w0 + other.y * w1;
            }
            const bool poisoned = *(const volatile int32_t *)&sg->poison != 0;
            const bool two = narrow && sg->nt > 1;   // slot 1 has an output to add
            const bool reject = *(const volatile bool *)&sg->reject;
            if (warp_live && (two || poisoned || reject)) {
                // what few outputs need is done to the output tile in tensor memory before it is written
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(tO + c, o);
                    tmem_wait_ld();
                    if (two) {
                        uint32_t o1[32];
                        tmem_ld32(tO + D + c, o1);
                        tmem_wait_ld();
                        // a slot whose keys this row does not see has weight 0 and a finite output
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            o[i] = __float_as_uint(__uint_as_float(o[i]) * w0 + __uint_as_float(o1[i]) * w1);
                    }
                    if (poisoned && live) {
                        // infinities and NaN among the values of the unit's own tokens, for the rows that see them
                        const int lo = max(sg->L + sg->first_token, sg->t0 * kKeyTile), hi = min(last_key, (sg->t0 + sg->nt) * kKeyTile - 1);
                        for (int key = lo; key <= hi; ++key) {
                            const int page = p.page_table[(size_t)sg->b * p.max_pages + key / kPage];
                            if (page < 0 || page >= p.num_pages) break;
                            const __nv_bfloat16 *v = v_pool + (((size_t)page * p.Hkv + sg->h) * kPage + key % kPage) * D + c;
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const float x = __bfloat162float(v[i]);
                                if (!isfinite(x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
                            }
                        }
                    }
                    if (reject) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0;
                    }
                    tmem_st32(tO + c, o);
                }
                tmem_wait_st();
            }
            if (warp_live) {
                const bool full = sg->full;
                const float inv = full && !reject ? 1.f / l_all : 1.f;
                const uint32_t staging = base + C::kOffStaging + warp * 4096;   // 32 rows of 128 bytes, 16-byte pieces swizzled
                // where this lane's row goes, in rows from the unit's first; -1: nowhere
                const int to = !live ? -1 : full ? unit_token * p.Hq + row_member : row;
                __nv_bfloat16 *out = p.out + (((size_t)sg->start + sg->first_token) * p.Hq + (size_t)sg->h * p.G) * D;
                float *part_o = p.partial_o + ((size_t)(2 * blockIdx.x + sg->slot) * 256 + slot * 128) * D;
                auto put = [&](int piece, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(staging + lane * 128 + ((piece ^ (lane & 7)) << 4)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
                };
                // eight lanes write a row's 128 bytes (64 bf16 or 32 fp32 columns), a warp four rows at a time
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(tO + c, o);
                    tmem_wait_ld();
                    if (full) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t y[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 hh = __floats2bfloat162_rn(__uint_as_float(o[8 * i + 2 * e]) * inv, __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
                                y[e] = *reinterpret_cast<const uint32_t *>(&hh);
                            }
                            put(((c >> 3) & 4) + i, y[0], y[1], y[2], y[3]);
                        }
                        if (!(c & 32)) continue;
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) put(i, o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                    }
                    char *rows = full ? reinterpret_cast<char *>(out + c - 32) : reinterpret_cast<char *>(part_o + c);
                    const int row_bytes = full ? D * 2 : D * 4;
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = i * 4 + (lane >> 3), piece = lane & 7;
                        const int dst = __shfl_sync(0xffffffffu, to, r);
                        uint4 y;
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w) : "r"(staging + r * 128 + ((piece ^ (r & 7)) << 4)));
                        if (dst >= 0) *reinterpret_cast<uint4 *>(rows + (size_t)dst * row_bytes + piece * 16) = y;
                    }
                    __syncwarp();
                }
                if (live) {
                    if (!sg->full)
                        *reinterpret_cast<float2 *>(p.partial_ml + ((size_t)(2 * blockIdx.x + sg->slot) * 256 + slot * 128 + row) * 2) = make_float2(m_all, l_all);
                    else if (p.lse)
                        p.lse[((size_t)sg->start + sg->first_token + unit_token) * p.Hq + (size_t)sg->h * p.G + row_member] = reject ? 0.f : (m_all + log2f(l_all)) * 0.6931471805599453f;
                }
            }
            if (narrow) {
                // slot 1's output has been read: its next product may overwrite it
                tc_fence_before();
                mbar_arrive(bar(&m->merge_free));
                ++narrows;
            }
            done();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
    const bool late = *abort_s || (int)blockIdx.x == p.give_up;
    if (tid == 0) p.gave_up[blockIdx.x] = late;
    const Piece &s = m->piece[0];
    if (p.alone && late && s.nt > 0) {   // (published before anything could be waited for)
        const int row_pieces = p.G * (D / 8);   // of the unit's heads of a token
        for (int i = tid; i < s.u.tokens * row_pieces; i += kThreads) {
            const size_t row = (size_t)(s.start + s.first_token + i / row_pieces) * p.Hq + (size_t)s.h * p.G;
            reinterpret_cast<uint4 *>(p.out + row * D)[i % row_pieces] = make_uint4(0, 0, 0, 0);
            if (p.lse && i % (D / 8) == 0) p.lse[row + i % row_pieces / (D / 8)] = 0.f;
        }
        if (tid == 0) note_late(p, s.b, (int)blockIdx.x - (s.block * p.Hkv + s.h));
    }
}

// After the attention kernel: blocks kMergeBlocks * c .. of the first n_ctas * kMergeBlocks merge the unit that CTA c
// began and others finished; the block of sequence b behind them reports it, zeroes its rows if it is rejected and
// advances its length.  A sequence's pages are checked here and not before the attention: an id outside the pool makes
// a tile load read the fill value, never a fault, and the rows computed with it are zeroed here.
//
// A merge is latency: a few kilobytes a row, spread over as many blocks and loads in flight as there are (with one block
// to a unit it took 30 us of a 52 us call).  A unit of few pieces has many rows: a warp takes a row (two at head_dim
// 64) and goes through the pieces; a unit of many pieces (few rows over a long history) gives a row's pieces to the
// eight warps of a block, which join their shares in shared memory.
constexpr int kFinishThreads = 256;
constexpr int kMergeBlocks = 8;

// This thread's share of a look at the pages of a sequence's first `keys` positions.
__device__ __forceinline__ bool sees_bad_page(const PromptAttnParams &p, int b, int keys) {
    bool bad = false;
    for (int i = threadIdx.x; i < (keys + kPage - 1) / kPage; i += kFinishThreads) {
        const int pg = p.page_table[(size_t)b * p.max_pages + i];
        bad |= pg < 0 || pg >= p.num_pages;
    }
    return bad;
}
__device__ __forceinline__ bool sees_late_cta(const PromptAttnParams &p) {
    bool late = false;
    for (int i = threadIdx.x; i < p.n_ctas; i += kFinishThreads) late |= p.gave_up[i] != 0;
    return late;
}

// Running softmax state of four columns of a row.
struct Merged {
    float mx, l, o[4];
    __device__ __forceinline__ void clear() {
        mx = -INFINITY;
        l = o[0] = o[1] = o[2] = o[3] = 0.f;
    }
    // A share with the maximum -inf has weight 0, not no weight: the row may see none of its keys (sum and output are 0), or
    // scores that are all NaN beside masked ones, which a maximum ignores and only the sum and the output tell.
    __device__ __forceinline__ void add(float m2, float l2, const float4 &y) {
        const float up = fmaxf(mx, m2), w = mx == -INFINITY ? 0.f : exp2f(mx - up), w2 = m2 == -INFINITY ? 0.f : exp2f(m2 - up);
        mx = up;
        l = l * w + l2 * w2;
        o[0] = o[0] * w + y.x * w2; o[1] = o[1] * w + y.y * w2; o[2] = o[2] * w + y.z * w2; o[3] = o[3] * w + y.w * w2;
    }
};

template <int D>
__device__ __forceinline__ void merge_unit(const PromptAttnParams &p, const PieceDesc &d, int c, int chunk) {
    constexpr int kLanes = D / 4, kRows = kFinishThreads / kLanes, kUnroll = 4;   // four columns a thread; rows at a time
    __shared__ float s_ml[8][2], s_o[8][D];
    const int tid = threadIdx.x;
    const UnitShape u = unit_shape(d.L, d.tokens, d.block, p.tile_tokens);
    const int tile_rows = p.tile_tokens * p.G, rows = u.tokens * p.G;
    auto place = [&](int k, int i) { return (size_t)(k == 0 ? 2 * c + 1 : 2 * (c + k)) * 256 + (i < tile_rows ? i : 128 + i - tile_rows); };
    auto write = [&](int i, int x, const Merged &m) {
        const float inv = 1.f / m.l;
        const int token = d.block * 2 * p.tile_tokens + i / p.G;
        const size_t row = (size_t)(d.first_token + token) * p.Hq + (size_t)d.h * p.G + i % p.G;
        const __nv_bfloat162 a = __floats2bfloat162_rn(m.o[0] * inv, m.o[1] * inv), b = __floats2bfloat162_rn(m.o[2] * inv, m.o[3] * inv);
        reinterpret_cast<uint2 *>(p.out + row * D)[x] = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
        if (p.lse && x == 0) p.lse[row] = (m.mx + log2f(m.l)) * 0.6931471805599453f;
    };
    if (d.more < 8) {
        const int x = tid % kLanes;
        for (int i0 = chunk + kMergeBlocks * (tid / kLanes); i0 < rows; i0 += kMergeBlocks * kRows * kUnroll) {
            Merged m[kUnroll];
#pragma unroll
            for (int r = 0; r < kUnroll; ++r) m[r].clear();
            for (int k = 0; k <= d.more; ++k) {
                float2 ml[kUnroll];
                float4 y[kUnroll];
#pragma unroll
                for (int r = 0; r < kUnroll; ++r) {
                    const int i = i0 + r * kMergeBlocks * kRows;
                    ml[r] = make_float2(-INFINITY, 0.f);
                    y[r] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (i < rows) {
                        ml[r] = *reinterpret_cast<const float2 *>(p.partial_ml + place(k, i) * 2);
                        y[r] = reinterpret_cast<const float4 *>(p.partial_o + place(k, i) * D)[x];
                    }
                }
#pragma unroll
                for (int r = 0; r < kUnroll; ++r) m[r].add(ml[r].x, ml[r].y, y[r]);
            }
#pragma unroll
            for (int r = 0; r < kUnroll; ++r)
                if (i0 + r * kMergeBlocks * kRows < rows) write(i0 + r * kMergeBlocks * kRows, x, m[r]);
        }
        return;
    }
    const int warp = tid >> 5, lane = tid & 31, x = lane % kLanes;
    for (int i = chunk; i < rows; i += kMergeBlocks) {
        Merged m;
        m.clear();
        for (int k0 = warp; k0 <= d.more; k0 += 8 * kUnroll) {
            float2 ml[kUnroll];
            float4 y[kUnroll];
#pragma unroll
            for (int r = 0; r < kUnroll; ++r) {
                ml[r] = make_float2(-INFINITY, 0.f);
                y[r] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k0 + 8 * r <= d.more) {
                    ml[r] = *reinterpret_cast<const float2 *>(p.partial_ml + place(k0 + 8 * r, i) * 2);
                    y[r] = reinterpret_cast<const float4 *>(p.partial_o + place(k0 + 8 * r, i) * D)[x];
                }
            }
#pragma unroll
            for (int r = 0; r < kUnroll; ++r) m.add(ml[r].x, ml[r].y, y[r]);
        }
        if (lane < kLanes) {
            if (lane == 0) {
                s_ml[warp][0] = m.mx;
                s_ml[warp][1] = m.l;
            }
            *reinterpret_cast<float4 *>(&s_o[warp][4 * x]) = make_float4(m.o[0], m.o[1], m.o[2], m.o[3]);
        }
        __syncthreads();
        if (warp == 0 && lane < kLanes) {
            Merged all;
            all.clear();
#pragma unroll
            for (int w = 0; w < 8; ++w) all.add(s_ml[w][0], s_ml[w][1], *reinterpret_cast<const float4 *>(&s_o[w][4 * x]));
            write(i, x, all);
        }
        __syncthreads();
    }
}

template <int D>
__global__ void __launch_bounds__(kFinishThreads) prompt_finish_kernel(const PromptAttnParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < p.n_ctas * kMergeBlocks) {
        const int c = blockIdx.x / kMergeBlocks;
        const PieceDesc d = p.pieces[c];
        const int chunk = blockIdx.x % kMergeBlocks;
        if (d.b < 0 || chunk >= unit_shape(d.L, d.tokens, d.block, p.tile_tokens).tokens * p.G) return;
        // (a rejected sequence's rows are zeroed below: nobody else may write them)
        if (!__syncthreads_or(sees_late_cta(p) || sees_bad_page(p, d.b, d.L + d.tokens))) merge_unit<D>(p, d, c, chunk);
        return;
    }
    const int b = blockIdx.x - p.n_ctas * kMergeBlocks;
    bool bad = false;
    for (int i = tid; i < p.B; i += kFinishThreads) {
        const int a = p.token_start[i], e = p.token_start[i + 1];
        bad |= a < 0 || a > e || e > p.tokens;
    }
    const int start = p.token_start[b], n = p.token_start[b + 1] - start, L = p.seq_lens[b];
    const bool len_ok = prompt_len_ok(L, n, p.max_pages);
    const bool page = len_ok && n > 0 && sees_bad_page(p, b, L + n), late = sees_late_cta(p);
    if (__syncthreads_or(bad)) {
        if (tid == 0) p.status[b] = READER_ERR_INVALID_ARG;
        return;   // whose rows are whose is not known: nothing was written
    }
    const bool any_page = __syncthreads_or(page), any_late = __syncthreads_or(late);
    const int st = !len_ok ? READER_ERR_CAPACITY : any_page ? READER_ERR_BAD_PAGE : any_late ? READER_ERR_TIMEOUT : READER_OK;
    if (tid == 0) {
        p.status[b] = st;
        if (p.bump && st == READER_OK) p.bump[b] = L + n;
    }
    if (st != READER_OK) zero_sequence(p, b, D, tid, kFinishThreads);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode(void *fn, CUtensorMap *map, const void *at, int rank, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box) {
    const cuuint32_t one[3] = {1, 1, 1};
    return reinterpret_cast<EncodeTiledFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(at), dims, strides, box, one,
                                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

reader_status launch_prompt_attn(bool *attr_set, void *fn, const PromptAttnParams &p, const __nv_bfloat16 *q, const void *k_pool,
                                 const void *v_pool, cudaStream_t st) {
    if (!*attr_set) {
        if (cudaFuncSetAttribute(prompt_attn_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<128>::kSmemBytes) != cudaSuccess ||
            cudaFuncSetAttribute(prompt_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<64>::kSmemBytes) != cudaSuccess) {
            cudaGetLastError();
            return READER_ERR_CUDA;
        }
        *attr_set = true;
    }
    // The descriptors are made anew for every call: about 0.1 us each, and nothing to go stale.
    alignas(64) CUtensorMap qmap, kmap, vmap;
    const cuuint64_t pool_dims[2] = {(cuuint64_t)p.D, (cuuint64_t)p.num_pages * p.Hkv * kPage}, pool_strides[1] = {(cuuint64_t)p.D * 2};
    const cuuint32_t pool_box[2] = {64, (cuuint32_t)kPage};
    // 64 columns x the G heads of a group x as many tokens as fill 128 rows
    const cuuint64_t q_dims[3] = {(cuuint64_t)p.D, (cuuint64_t)p.Hq, (cuuint64_t)p.tokens};
    const cuuint64_t q_strides[2] = {(cuuint64_t)p.D * 2, (cuuint64_t)p.Hq * p.D * 2};
    const cuuint32_t q_box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.tile_tokens};
    if (!encode(fn, &kmap, k_pool, 2, pool_dims, pool_strides, pool_box) || !encode(fn, &vmap, v_pool, 2, pool_dims, pool_strides, pool_box) ||
        !encode(fn, &qmap, q, 3, q_dims, q_strides, q_box))
        return READER_ERR_CUDA;
    const bool wide = p.D == 128;
    const cudaError_t e = launch_pdl(wide ? prompt_attn_kernel<128> : prompt_attn_kernel<64>, dim3((unsigned)p.n_ctas), dim3(kThreads),
                                     wide ? Cfg<128>::kSmemBytes : Cfg<64>::kSmemBytes, st, p, qmap, kmap, vmap,
                                     static_cast<const __nv_bfloat16 *>(v_pool));
    if (e != cudaSuccess) {
        cudaGetLastError();
        return READER_ERR_CUDA;
    }
    return READER_OK;
}

void launch_prompt_finish(const PromptAttnParams &p, cudaStream_t st) {
    launch_pdl(p.D == 128 ? prompt_finish_kernel<128> : prompt_finish_kernel<64>, dim3((unsigned)(p.n_ctas * kMergeBlocks + p.B)), dim3(kFinishThreads), 0, st, p);
}

}  // namespace reader

// Parameter block and work partition of the prompt attention (reader_prompt_attn).
#pragma once
#include "common.cuh"

namespace reader {

constexpr int kPromptMaxBatch = 32768;   // the partition of a call is worked out in shared memory, one word per sequence
constexpr int kKeyTile = 128;            // keys per tile: two cache pages

// A unit is (sequence, KV head, block of 2 * tile_tokens consecutive new tokens): up to 256 query rows, row
// = token * G + group member within each of two 128-row tiles.
//   wide unit    both tiles have rows: a step is one key tile, multiplied with both query tiles
//   narrow unit  only the first tile has rows (the last block of a sequence, every block of a single-token call):
//                a step is two key tiles, each multiplied with the one query tile, merged at the unit's end
// A call with many units hands them out whole, from a counter.  Otherwise the units in the order (sequence, KV head,
// block), each kUnitEntries entries (what starting and ending a unit costs) followed by its steps, form one list that is
// cut into contiguous equal ranges, one per CTA.
// Measured, us at 32/8/128 heads.  kUnitEntries 1, 2, 4: a prompt of 1500 tokens 52, 54, 57 (runs differ by 5 %), of 2500 90, 87,
// 92; two pieces on 30 k histories 939, 928, 946; 16 pieces of 1 to 300 on 500 to 3000 120, 120, 126.  kNarrowUnitEntries 0, 1, 3
// (a narrow unit's loads run on from the unit before it): 32 single tokens on 1024 to 4096 74.6, 71.1, 70.5; 8 x 16 tokens
// on 2000 to 4000 35.6, 35.0, 35.4.  kMinEntriesPerCta 2, 4, 8: one token on 16000 24.9, 23.4, 35.1; four on 1000 to 2000
// 21.2, 23.8, 31.5; calls with entries for every CTA do not notice.
constexpr int kUnitEntries = 2;
constexpr int kNarrowUnitEntries = 1;
constexpr int kMinEntriesPerCta = 4;
// A call is a single launch when its units fit the CTAs and cutting them would not pay for the merge and the second launch
// (6 to 9 us): going by the page table's width, at most kAloneSteps steps to a unit (lengths may differ, and the longest
// one decides), and at most kAloneIdle steps that a CTA would gain on average from the CTAs without a unit.  Measured, alone
// against cut: one token on 1000, 1500, 2000 keys, 8 units: 15.9 / 21.3, 20.0 / 19.8, 24.1 / 20.4 us; 16 tokens on 1500
// keys each, 128 units: 24.8 / 34.6 us; a prompt of 1500 tokens in 24 units: 35.0 / 30.4 us, of 1000 in 128: 24.5 / 34.2 us.
// The host does not know the lengths: one token on 511 keys takes 9.6 us behind a table of 8 pages and 19.4 behind one of 32
// or of 2048, where the call is cut; and a call that advances the lengths is never alone.
constexpr int kAloneSteps = 12, kAloneIdle = 6;
// Units per CTA from which a call hands them out from a counter (a prompt of 4096 tokens, 3.5 units per CTA: 158 us, cut into
// equal ranges 167 us; 16 prompts, 16 units per CTA: 314 and 340 us).  Here too it is the tensors' rows that count, not the
// tokens in them: 32 single tokens on 1024 to 4000 keys take 69 us in a call made for 32 rows and 75 in one made for 4096;
// one token on 30000, which the counter does not cut, 32 and 241 us.
constexpr int kDynamicUnits = 3;

struct PieceDesc {        // a unit that CTA c starts but does not finish: pieces 2c + 1, then 2(c + 1), 2(c + 2), ...
    int32_t b, h, block;  // b = -1: none
    int32_t more;         // how many CTAs follow
    int32_t first_token, tokens, L;
};

struct PromptAttnParams {
    const int32_t *token_start;   // [B + 1]
    const int32_t *seq_lens, *page_table;
    int B, tokens, Hq, Hkv, G, D, max_pages, num_pages;
    int shared_prefix_len;
    int tile_tokens;              // tokens per 128-row tile: 128 / G, rounded down
    float scale_log2;
    __nv_bfloat16 *out;
    float *lse;
    int32_t *status;
    int32_t *bump;                // seq_lens again when it is to be advanced, else null
    int n_ctas;
    int32_t *counter;             // next unit to hand out, zero at the start; null: the units are dealt out beforehand
    bool alone;                   // at most one unit per CTA, each done whole, and no finishing kernel behind
    // workspace
    float *partial_o;             // [2 n_ctas][256][D]
    float *partial_ml;            // [2 n_ctas][256][2]
    PieceDesc *pieces;            // [n_ctas]
    int32_t *gave_up;             // [n_ctas]
    uint64_t *late_notes;         // [n_ctas], single-launch form: kLateNote in the word of a sequence's first unit, see note_late
    int give_up;                  // a CTA that says it gave up when it is done (testing aid); -1: none
};
constexpr uint64_t kLateNote = 0x9d6b2f04c18e73a5ull;   // (the workspace holds anything beforehand)

// Whether a sequence takes part: what the host cannot check and the partition depends on.
__host__ __device__ inline bool prompt_len_ok(int L, int n, int max_pages) {
    return n >= 0 && L >= 0 && (int64_t)L + n <= (int64_t)max_pages * kPage;
}

struct UnitShape {
    int tokens;     // new tokens in the block
    int keys;       // keys its last token sees
    bool narrow;
    int tiles, steps;
    __host__ __device__ int entries() const { return (narrow ? kNarrowUnitEntries : kUnitEntries) + steps; }
};
__host__ __device__ inline UnitShape unit_shape(int L, int n, int block, int tile_tokens) {
    UnitShape u;
    const int first = block * 2 * tile_tokens;
    u.tokens = n - first < 2 * tile_tokens ? n - first : 2 * tile_tokens;
    u.keys = L + first + u.tokens;
    u.narrow = u.tokens <= tile_tokens;
    u.tiles = (u.keys + kKeyTile - 1) / kKeyTile;
    u.steps = u.narrow ? (u.tiles + 1) / 2 : u.tiles;
    return u;
}
__host__ __device__ inline int unit_blocks(int n, int tile_tokens) { return (n + 2 * tile_tokens - 1) / (2 * tile_tokens); }

// CTAs that share a list of W entries, where a CTA's range begins, and whose entry x is.
__host__ __device__ inline int prompt_busy_ctas(int n_ctas, int W) {
    const int want = (W + kMinEntriesPerCta - 1) / kMinEntriesPerCta;
    return want < 1 ? 1 : want < n_ctas ? want : n_ctas;
}
__host__ __device__ inline int prompt_range_begin(int c, int W, int ctas) { return (int)((int64_t)c * W / ctas); }
__host__ __device__ inline int prompt_range_owner(int x, int W, int ctas) { return (int)((((int64_t)x + 1) * ctas - 1) / W); }

// `attr_set`: whether the kernels have their shared-memory limit yet; `encode_tiled`: the driver's tensor-map encoder.
reader_status launch_prompt_attn(bool *attr_set, void *encode_tiled, const PromptAttnParams &p, const __nv_bfloat16 *q,
                                 const void *k_pool, const void *v_pool, cudaStream_t st);
void launch_prompt_finish(const PromptAttnParams &p, cudaStream_t st);

}  // namespace reader

// A page of keys or values in 4 bits.
//
// Numbers.  16 consecutive elements of one head of one position (a block) share a scale
//     s(c) = (1 + (c & 7) / 8) 2^((c >> 3) - 18),   c = 0 .. 254,
// the smallest with 7.5 s >= the block's largest magnitude (the largest scale if there is none), and every element x is
// held as n = q + 8, where q is x / s rounded to the nearest whole number (ties to even) and kept within -7 .. 7: no element
// is off by more than s / 2 (a magnitude above 7.5 s(254) = 107520 excepted).  c = 255 stands for a block with an
// infinity or a NaN and reads as NaN.  A value q s has at most 3 + 4 significant bits, so bf16 holds it exactly: attention
// over the values is the attention over a bf16 cache that holds them, with no rounding of its own.
// (Uniform numbers rather than a 4-bit float: on normal data a block of 16 is 2 dB closer to its input, 22.7 instead of 20.8,
// and a pair of numbers becomes a pair of bf16 in 2.75 instructions.)
//
// Places.  One (page, KV head) is a tile of 36 D bytes: 32 D of numbers, then 4 D of scales.  Eight numbers make a 32-bit word,
// a pair (low, high half of a future bf16 pair) per step i = 0 .. 3: low number i at bits 4 i, high number i at bits 16 + 4 i, and
// the word is rotated left by three bits, so that after a rotation right by 4 i the pair i stands in the lower bits of two bf16
// mantissas.
//   keys    word w of position r (at r D / 8 + w): elements 8 w .. 8 w + 7, the even ones low, the odd ones high
//   values  word y of the position pair t = r / 2 (row t of D / 4 words): elements 4 y .. 4 y + 3, position 2 t low, 2 t + 1
//           high; the row's eight chunks of D / 32 words are permuted (v_chunk) against shared-memory bank conflicts
//   scales  in the order in which the 32 lanes of a warp use them as fragments of a matrix product (k_scale_at, v_scale_at)
#pragma once
#include "common.cuh"

namespace reader {
namespace q4 {

constexpr int kBlock = 16;         // elements that share a scale
constexpr int kMaxCode = 254;      // largest scale
constexpr int kNanCode = 255;
constexpr int kScaleBias = 18;

__host__ __device__ constexpr int tile_bytes(int D) { return 36 * D; }
__host__ __device__ constexpr int scales_at(int D) { return 32 * D; }

template <int D>
__device__ __forceinline__ int k_scale_at(int r, int u) {
    constexpr int kPer = D / 64;   // blocks of a lane: lane 4 (r mod 8) + u / kPer
    return (((r & 7) * 4 + u / kPer) * 8 + (r >> 3)) * kPer + u % kPer;
}
template <int D>
__device__ __forceinline__ int v_scale_at(int r, int u) {
    return ((u * 4 + ((r >> 1) & 3)) * 8 + (r >> 3)) * 2 + (r & 1);
}
template <int D>
__device__ __forceinline__ int v_chunk(int t, int chunk) {
    return chunk ^ (D == 128 ? 2 * (t & 3) : 4 * ((t >> 1) & 1));
}

__device__ __forceinline__ float scale_of(int code) {
    return code == kNanCode ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(code + ((127 - kScaleBias) << 3)) << 20);
}

// The scale code of a block whose largest magnitude is the bf16 with these bits (finite, no sign).  Where it is (128 + t) / 128 2^e, the smallest m
// with 7.5 (8 + m) / 8 2^(e - 3) no less has 15 (8 + m) >= 128 + t; m of 8 and 9 carry into the exponent and mean the scales they should.
__device__ __forceinline__ int code_of(uint32_t top) {
    const int e = (int)(top >> 7) - 127, t = top & 127;
    return max(0, min(kMaxCode, (e - 3 + kScaleBias) * 8 + (128 + t + 14) / 15 - 8));
}

// 1 / s to within a unit in the last place or so.
__device__ __forceinline__ float reciprocal(float s) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return r;
}
// Two bf16, each brought into least .. most.
__device__ __forceinline__ uint32_t bf16x2_within(uint32_t x, uint32_t least, uint32_t most) {
    uint32_t d;
    asm("{\n\t.reg .b32 t;\n\tmax.bf16x2 t, %1, %2;\n\tmin.bf16x2 %0, t, %3;\n\t}" : "=r"(d) : "r"(x), "r"(least), "r"(most));
    return d;
}

__device__ __forceinline__ uint32_t turned(uint32_t plain) { return __funnelshift_l(plain, plain, 3); }
__device__ __forceinline__ uint32_t plain_of(uint32_t word) { return __funnelshift_r(word, word, 3); }

struct Block {   // 16 elements
    uint32_t n[2];   // of eight elements each
    int code;
};

// raw: 16 bf16.  Element e stands at bits 4 (e mod 8) of n[e / 8], or (kEvensApart) at 4 (e mod 8) / 2, odd ones 16 higher.
// A number is x / s to the nearest whole one, ties to even, plus 8.  x * (1 / s) may miss a tie by some units in the last place; one
// correction with the remainder, which an fma gives without rounding, makes it the quotient (to 2^-44, so exactly where that is a float).  Elements beyond 7 s (a bf16) are
// that first: 7.5 s would become 8.  Added to 1.5 * 2^23 + 8 the numbers stand in the lowest bits of floats, and sixteen times one of them plus the next, as whole
// numbers, is a shift and an or; what is above the numbers adds up to a constant.  (12 instructions for an element before, 6 now: a kernel
// that stores was bound by them.)
template <bool kEvensApart>
__device__ __forceinline__ Block quantise(const uint4 &a, const uint4 &b) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t tops = 0;   // magnitudes compare as whole numbers; infinity and NaN are the largest
#pragma unroll
    for (int i = 0; i < 8; ++i) tops = __vmaxu2(tops, w[i] & 0x7fff7fffu);
    const uint32_t top = max(tops << 16, tops & 0xffff0000u);
    Block r;
    if (top >= 0x7f800000u) {
        r.code = kNanCode;
        r.n[0] = r.n[1] = 0x88888888u;
        return r;
    }
    r.code = code_of(top >> 16);
    const float s = scale_of(r.code), inv = reciprocal(s);
    const uint32_t most = (__float_as_uint(7.f * s) >> 16) * 0x10001u, least = most | 0x80008000u;
    const float2 minus_s = make_float2(-s, -s), inv2 = make_float2(inv, inv), base = make_float2(12582920.f, 12582920.f);
    constexpr uint32_t kAbove = 0x4b400000u * 0x11111111u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = bf16x2_within(w[4 * h + i], least, most);
            const float2 x = make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
            float2 y = __fmul2_rn(x, inv2);
            y = __ffma2_rn(__ffma2_rn(y, minus_s, x), inv2, y);
            y = __fadd2_rn(y, base);
            lo[i] = __float_as_uint(y.x);
            hi[i] = __float_as_uint(y.y);
        }
        uint32_t n = 0;
        if (kEvensApart) {
#pragma unroll
            for (int i = 3; i >= 0; --i) n = n * 16u + hi[i];
#pragma unroll
            for (int i = 3; i >= 0; --i) n = n * 16u + lo[i];
        } else {
#pragma unroll
            for (int i = 3; i >= 0; --i) n = (n * 16u + hi[i]) * 16u + lo[i];
        }
        r.n[h] = n - kAbove;
    }
    return r;
}

// Back from evens apart: a word's eight numbers in the elements' order.
__device__ __forceinline__ uint32_t in_order(uint32_t w) {
    uint32_t e = w & 0xffffu, o = w >> 16;
    e = (e | (e << 8)) & 0x00ff00ffu;
    o = (o | (o << 8)) & 0x00ff00ffu;
    e = (e | (e << 4)) & 0x0f0f0f0fu;
    o = (o | (o << 4)) & 0x0f0f0f0fu;
    return e | (o << 4);
}

// Eight elements' values as bf16.
__device__ __forceinline__ uint4 values_of(uint32_t n, float s) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = ((int)((n >> (8 * i)) & 15u) - 8) * s, hi = ((int)((n >> (8 * i + 4)) & 15u) - 8) * s;
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        w[i] = *reinterpret_cast<const uint32_t *>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Block u of position r of a key tile (evens apart).
template <int D>
__device__ __forceinline__ void put_key_block(unsigned char *tile, int r, int u, const Block &b) {
    uint2 w;
    w.x = turned(b.n[0]);
    w.y = turned(b.n[1]);
    *reinterpret_cast<uint2 *>(tile + r * (D / 2) + u * 8) = w;
    tile[scales_at(D) + k_scale_at<D>(r, u)] = (unsigned char)b.code;
}

// Block u of a position pair of a value tile (in order): one of the two or both; the other keeps what it is.
template <int D>
__device__ __forceinline__ void put_value_blocks(unsigned char *tile, int t, int u, bool has_even, const Block &even, bool has_odd,
                                                 const Block &odd) {
    // four elements' numbers are 16 bits: word y = even half | odd half
    uint32_t w[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        const int sh = 16 * (y & 1);
        w[y] = turned(((even.n[y >> 1] >> sh) & 0xffffu) | (((odd.n[y >> 1] >> sh) & 0xffffu) << 16));
    }
    constexpr int kChunkWords = D / 32;   // a block is one chunk of four words, or two neighbouring ones of two
    const int chunk = v_chunk<D>(t, u * (4 / kChunkWords));
    uint4 *at = reinterpret_cast<uint4 *>(tile + t * D + chunk * kChunkWords * 4);
    unsigned char *scale = tile + scales_at(D) + v_scale_at<D>(2 * t, u);
    if (has_even && has_odd) {
        *at = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint16_t *>(scale) = (uint16_t)(even.code | (odd.code << 8));
        return;
    }
    const uint32_t mine = turned(has_even ? 0x0000ffffu : 0xffff0000u);
    const uint4 was = *at;
    *at = make_uint4((was.x & ~mine) | (w[0] & mine), (was.y & ~mine) | (w[1] & mine), (was.z & ~mine) | (w[2] & mine), (was.w & ~mine) | (w[3] & mine));
    scale[has_even ? 0 : 1] = (unsigned char)(has_even ? even.code : odd.code);
}

}  // namespace q4
}  // namespace reader

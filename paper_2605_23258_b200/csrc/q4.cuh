// Rows in microscaled 4-bit floating point, and the pages that hold them.
//
// A group of 16 neighbouring channels shares a scale s, an unsigned number of five exponent bits (bias 15) and three mantissa
// bits; a channel is one of {0, 1/2, 1, 3/2, 2, 3, 4, 6} s with its sign (e2m1).  s is the smallest with 6 s >= max |x|, so that
// nothing is cut off, and the channel's code the nearest, ties to the even code.  A scale's byte shifted left by seven is the same
// number in fp16, and a code times a scale has at most six significant bits: what a row stands for is exact in fp16 (and in bf16),
// one conversion and one product for two channels, and a product with it on the tensor cores is exact.  The scale goes up to 10240, so that
// 6 s stays within fp16; larger rows are cut off there.  Exponent 31 is not a number, as in fp16: a group with a NaN in it reads as NaN.
//
// A page holds 64 rows for every (layer, KV head): tiles of 64 rows of D / 2 bytes of codes, then 64 rows of D / 16 scales
// (72 bytes a row at 128 channels).  Order of a row: four pieces; piece t has the channels [t D/8, (t+1) D/8) and then those half a head above
// them, low nibble first, and the scales follow the same order.  A piece is what one lane of a quad reads as its part of a warp's
// 16 x 16 matrix fragments, and a rotary pair lies within it.
#ifndef VECTOR_Q4_CUH_
#define VECTOR_Q4_CUH_

#include "common.cuh"
#include "tcgen05.cuh"
#include "vector.h"

namespace vec {
namespace q4 {

constexpr int ROWS = VECTOR_PAGE_ROWS;
constexpr int SCALE_TOP = 226;                 // code of 10240
constexpr int SCALE_NAN = 255;
// Most pages of a pool: slots are 32-bit numbers.
constexpr int64_t MAX_PAGES = int64_t(1) << 25;

template <int D> struct Row {
    static constexpr int CODES = D / 2, GROUPS = D / 16;
    static constexpr int TILE = ROWS * (CODES + GROUPS);
    static constexpr int SCALES_AT = ROWS * CODES;                    // within a tile
    // Byte of a channel's code within its row, and place of a group's scale.
    __host__ __device__ static constexpr int byte_of(int c) { return ((c % (D / 2)) / (D / 8) * (D / 4) + c / (D / 2) * (D / 8) + c % (D / 8)) / 2; }
    __host__ __device__ static constexpr int scale_of(int group) { return 2 * (group % (D / 32)) + group / (D / 32); }
    // The channel of element e (nibble e & 1 of byte e / 2) of a row.
    __host__ __device__ static constexpr int channel_of(int e) { return e / (D / 4) * (D / 8) + e % (D / 4) / (D / 8) * (D / 2) + e % (D / 8); }
};

__device__ __forceinline__ float scale_value(uint32_t code) { return __half2float(__ushort_as_half((unsigned short)(code << 7))); }

// The smallest scale with 6 s >= most.  The product below is under most / 6 by 2^-22 to 2^-21 of it: truncated, it is the scale sought,
// or one or two below; 6 s is exact, so the comparisons are.
__device__ __forceinline__ uint32_t scale_code(float most) {
    if (!(most <= 3.4e38f)) return most != most ? (uint32_t)SCALE_NAN : (uint32_t)SCALE_TOP;
    uint32_t c = (uint32_t)__half_as_ushort(__float2half_rz(most * 0.16666663f)) >> 7;
    c += 6.f * scale_value(c) < most;
    c += 6.f * scale_value(c) < most;
    return min(c, (uint32_t)SCALE_TOP);
}

// Eight numbers to their codes, the first in the lowest nibble.
__device__ __forceinline__ uint32_t to_codes(const float (&q)[8]) {
    uint32_t r;
    asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}\n"
        : "=r"(r) : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
    return r;
}
// The quotients x / s are on the right side of every border between codes.  A border is t s, t of at most three significant bits.
// bf16: x has eight bits and t s seven, so x is t s or at least 2^-8 of it away, which no rounding below crosses; and where x = t s the quotient has to be t: 1 / s enters in
// two parts, so that what is left of x / s is under 2^-40 of it and the last rounding gives t.
__device__ __forceinline__ uint2 encode_group(const uint4 (&v)[2], uint32_t& scale) {
    uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
    uint32_t most = w[0] & 0x7fff7fffu;                                // magnitudes order like their bits, NaN above all
#pragma unroll
    for (int i = 1; i < 8; ++i) asm("max.u16x2 %0, %0, %1;\n" : "+r"(most) : "r"(w[i] & 0x7fff7fffu));
    scale = scale_code(__uint_as_float(max(most << 16, most & 0xffff0000u)));
    if (scale >= SCALE_TOP) {                                          // infinities count as the largest number
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t size = w[i] & 0x7fff7fffu;
            asm("min.u16x2 %0, %0, %1;\n" : "+r"(size) : "r"(0x7f7f7f7fu));
            w[i] = size | (w[i] & 0x80008000u);
        }
    }
    const float s = scale_value(scale), inv = s > 0.f ? __frcp_rn(s) : 0.f, rest = fmaf(-inv, s, s > 0.f ? 1.f : 0.f) * inv;
    const uint64_t inv2 = tc::pack2(inv, inv), rest2 = tc::pack2(rest, rest);
    uint32_t codes[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t x = tc::pack2(__uint_as_float(w[4 * h + i] << 16), __uint_as_float(w[4 * h + i] & 0xffff0000u));
            tc::unpack2(tc::fma2(x, inv2, tc::mul2(x, rest2)), q[2 * i], q[2 * i + 1]);
        }
        codes[h] = to_codes(q);
    }
    return make_uint2(codes[0], codes[1]);
}
// fp32: the quotient rounded to twelve bits (h s is exact then), moved by one unit in the last place to the side that what is left, x - h s, says.
__device__ __forceinline__ float quotient_f32(float x, float s, float inv) {
    const uint32_t h = (__float_as_uint(x * inv) + 0x800u) & 0xfffff000u;
    const float left = fmaf(-__uint_as_float(h), s, x);
    const bool out = (__float_as_uint(left) ^ h) >> 31 == 0;           // away from zero
    return __uint_as_float(h + (left > 0.f || left < 0.f ? (out ? 1u : 0xffffffffu) : 0u));
}
__device__ __forceinline__ uint2 encode_group(const uint4 (&v)[4], uint32_t& scale) {
    uint32_t x[16], most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[4 * i] = v[i].x; x[4 * i + 1] = v[i].y; x[4 * i + 2] = v[i].z; x[4 * i + 3] = v[i].w; }
#pragma unroll
    for (int i = 0; i < 16; ++i) most = max(most, x[i] & 0x7fffffffu);
    scale = scale_code(__uint_as_float(most));
    const float s = scale_value(scale), inv = s > 0.f ? __frcp_rn(s) : 0.f;
    uint32_t codes[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = quotient_f32(__uint_as_float(x[8 * h + i]), s, inv);
        codes[h] = to_codes(q);
    }
    return make_uint2(codes[0], codes[1]);
}

// The eight codes of a word as four fp16 pairs, before the scale.
__device__ __forceinline__ void decode_word(uint32_t w, uint32_t (&p)[4]) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
        : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3]) : "r"(w));
}

}  // namespace q4
}  // namespace vec
#endif

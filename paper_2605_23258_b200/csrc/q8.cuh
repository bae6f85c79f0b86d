// Rows in 8 bits, and the pages that hold them.
//
// A channel is an e4m3 number (sign, four exponent bits of bias 7, three mantissa bits, largest 448, no infinities) times 2^e, and a block of 32 tokens of one
// (layer, KV head), its keys or its values, shares e: the smallest in [-32, 31] with 448 2^e >= max |x|.  Numbers within 2^14 of the block's largest keep their
// four significant bits, so outlier channels cost the others nothing, and a power of two leaves the products of a block of rows exact: attention takes a row as
// fp16 (one conversion for two channels, exact), and the factor once for a block.  Why one scale for many tokens: with a floating format it only has to put the
// block into range; a scale a group of channels, as in the 4-bit pages, would cost a product for two channels in attention.  What is larger than 448 2^31 is
// cut off there, infinities too; a NaN stays one channel's NaN and does not count for the scale.
//
// A page is such a block: for every (layer, KV head) a tile of 32 rows of D bytes, then 32 bytes of which the first is e + 32.  Order of a row: what lane t of
// a quad holds of a warp's 16 x 16 matrix fragments is channels [t D/8, (t+1) D/8) and those half a head above them.  128 channels: as they are, but the halves
// of odd rows change places, so that the quads of two rows that read 16 bytes a lane at once meet in no bank.  64 channels: a lane's two runs of eight bytes
// lie together.
#ifndef VECTOR_Q8_CUH_
#define VECTOR_Q8_CUH_

#include "common.cuh"
#include "vector.h"

namespace vec {
namespace q8 {

constexpr int ROWS = VECTOR_Q8_PAGE_ROWS;
constexpr int LOW = -32, HIGH = 31;            // exponents of a scale
constexpr int64_t MAX_PAGES = int64_t(1) << 26;        // of a pool: places of rows are 32-bit numbers

template <int D> struct Row {
    static constexpr int TILE = ROWS * D + 32, SCALE_AT = ROWS * D;
    // Byte of a channel within its row.  Runs of 64 (128 channels) or 8 stay together.
    __host__ __device__ static constexpr int byte_of(int row, int c) {
        return D == 128 ? ((c / 64) ^ (row & 1)) * 64 + c % 64 : c % 32 / 8 * 16 + c / 32 * 8 + c % 8;
    }
};

// 2^e for e in [-126, 127].
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// The exponent for a largest magnitude, as the bits of an fp32 number that is no NaN.
__device__ __forceinline__ int exponent(uint32_t most) {
    const int e = (int)(most >> 23) - 127 - 8 + ((most & 0x7fffffu) > 0x600000u);        // 448 = 1.75 2^8
    return min(max(e, LOW), HIGH);
}
// A tile's exponent; what is no code of one (a page that nobody wrote) counts as the largest.
__device__ __forceinline__ int exponent_of(const unsigned char* tile, int scale_at) { return min((int)tile[scale_at], HIGH - LOW) + LOW; }

// Four numbers to their codes, the first in the lowest byte; 448 is where larger ones are cut off.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    uint32_t r;
    asm("{\n .reg .b16 lo, hi;\n cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n mov.b32 %0, {lo, hi};\n}\n"
        : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}
// The four codes of a word as two fp16 pairs, exact.
__device__ __forceinline__ void decode_word(uint32_t w, uint32_t& p0, uint32_t& p1) {
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n cvt.rn.f16x2.e4m3x2 %1, hi;\n}\n" : "=r"(p0), "=r"(p1) : "r"(w));
}
__device__ __forceinline__ void decode_word(uint32_t w, float (&x)[4]) {
    uint32_t p0, p1;
    decode_word(w, p0, p1);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&p0)), b = __half22float2(*reinterpret_cast<const __half2*>(&p1));
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

}  // namespace q8
}  // namespace vec
#endif

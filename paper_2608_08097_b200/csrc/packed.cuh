// The packed entry: keys and values of one (block, KV head) in 4 bits, 2,304 bytes instead of 8,192.
//
//   [0, 1024)      key codes: dims 32c .. 32c + 31 of token i in 16 bytes at 256 c + 16 i
//   [1024, 2048)   value codes: the 16 tokens of dim d in 8 bytes at 1024 + 8 d
//   [2048, 2176)   key scales: one byte for dims 16g .. 16g + 15 of token i at 2048 + 8 i + g
//   [2176, 2304)   value scales: one byte for the 16 tokens of dim d at 2176 + d
// Eight codes are a 32-bit word: code 2p in bits 4p .. 4p + 3, code 2p + 1 in bits 16 + 4p .. 16 + 4p + 3, so that one shift and one
// three-input logic instruction put two neighbours into the halves of a register.  A code c stands for (c - 8) * s, a scale byte b
// for s = (1 + (b & 7) / 8) * 2^((b >> 3) - 20): a sign-less float of five exponent and three fraction bits, no zero.
//
// Why these: both products of the attention run over bf16 operands.  |c - 8| <= 8 has four significant bits and s has four, so
// (c - 8) * s is exact in bf16 and the attention adds no rounding of its own to the quantisation.  Whole numbers at equal distances lose less than 4-bit floats on groups as small as 16: 8.6 %
// of the norm of normally distributed values.  The groups follow the attention's operands: a thread that prepares keys owns a
// token, one that prepares values a dim, and each of its sixteen values share a scale.
#pragma once
#include "common.cuh"

namespace oasis {

constexpr int kPackedBytes = OASIS_PACKED_BYTES;
constexpr int kPackedV = 1024, kPackedKScale = 2048, kPackedVScale = 2176;
constexpr int kScaleBias = 20;

// The scale byte of a group whose largest magnitude is `amax` (not NaN): amax / 7, to four significant bits, ties to even.
// (amax has 8 bits: where the exact quotient is a tie the rounded one is too, elsewhere it is 2^-9 away from one.)
__device__ __forceinline__ int scale_byte(float amax)
{
    const uint32_t u = __float_as_uint(__fdiv_rn(amax, 7.0f));
    const int byte = (int)((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - ((127 - kScaleBias) << 3);
    return min(max(byte, 0), 255);
}
__device__ __forceinline__ float scale_value(int byte) { return __uint_as_float(((uint32_t)byte << 20) + ((127u - kScaleBias) << 23)); }
// What `code_bits` multiplies by: 1 / s, a little less.  Products are then below the exact quotient by 2^-21 to 2^-19 of it, so that
// a value halfway between two multiples of s goes to the smaller one; any other quotient is 2^-9 of itself from a halfway point.
__device__ __forceinline__ float scale_inverse(int byte) { return __fdiv_rn(1.0f - 0x1p-20f, scale_value(byte)); }
// c = 8 + the nearest whole number to x / s within +-7, in the low bits (x is not NaN).
__device__ __forceinline__ uint32_t code_bits(float x, float inv)
{
    return __float_as_uint(fminf(fmaxf(x * inv, -7.0f), 7.0f) + 12582920.0f) & 15u;
}

// Eight codes of a word as four bf16 pairs (c - 8) * s * 2^-kDequantShift.  A whole number n < 256 in the low bits of a bf16 is
// n * 2^-133 (subnormal up to 127, and the first binade has the same spacing): so a nibble in bits 0 .. 3 needs no more than a mask
// to be c * 2^-133, one in bits 4 .. 7 c * 2^-129, and one shift serves the other two pairs.  A fused multiply-add takes the power of
// two, the scale and the 8 away; the shift keeps its factor below 2^128.
constexpr int kDequantShift = 20;
struct DequantScale {
    uint32_t lo, hi, minus;                            // (x, x) for s 2^(133 - shift), s 2^(129 - shift), -8 s 2^-shift
};
// `twice`: the scale byte in both halves (0x00bb00bb).
__device__ __forceinline__ DequantScale dequant_scale(uint32_t twice)
{
    DequantScale d;
    d.lo = twice * 16u + 0x00010001u * ((127u - kScaleBias + 133u - kDequantShift) << 7);
    d.hi = twice * 16u + 0x00010001u * ((127u - kScaleBias + 129u - kDequantShift) << 7);
    d.minus = twice * 16u + 0x00010001u * (0x8000u | ((127u - kScaleBias + 3u - kDequantShift) << 7));
    return d;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ void dequant_word(uint32_t w, const DequantScale &d, uint32_t *out)
{
    const uint32_t v = w >> 8;
    out[0] = fma_bf16x2(w & 0x000f000fu, d.lo, d.minus);
    out[1] = fma_bf16x2(w & 0x00f000f0u, d.hi, d.minus);
    out[2] = fma_bf16x2(v & 0x000f000fu, d.lo, d.minus);
    out[3] = fma_bf16x2(v & 0x00f000f0u, d.hi, d.minus);
}

}  // namespace oasis

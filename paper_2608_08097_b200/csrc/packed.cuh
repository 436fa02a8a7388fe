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

// The scale byte of a group whose largest magnitude has the bf16 pattern `amax` (at most kPackLargest): amax / 7 to four significant
// bits, ties to even.  With amax = (128 + M) 2^(E - 134) that is 8 (E - 110) + scale_step(M): M's 128 values are a table that the warp
// holds in a register, four bytes a lane.
constexpr uint32_t kPackLargest = 0x46d2;              // 26880 = 7 * 3840, the largest value that the largest scale reaches
template <uint32_t UNIT>
__host__ __device__ constexpr uint32_t nearest_even(uint32_t x)        // x / UNIT, ties to even
{
    return x / UNIT + (2 * (x % UNIT) > UNIT || (2 * (x % UNIT) == UNIT && x / UNIT % 2 == 1) ? 1 : 0);
}
__host__ __device__ constexpr uint32_t scale_step(uint32_t m)
{
    // (128 + M) / 7 lies in [16, 37): 8 .. 16 units of 2 below 32, 8 or 9 of 4 from there on
    return m < 96 ? nearest_even<14>(128 + m) - 8 : nearest_even<28>(128 + m);
}
static_assert(scale_step(0) == 1 && scale_step(133 - 128) == 2 && scale_step(147 - 128) == 2 && scale_step(96) == 8 && scale_step(238 - 128) == 8, "scale steps");
struct PackTables {
    uint32_t steps[32];                                // four scale_step() each
    float inverses[8];                                 // 2^-20 less than 8 / (8 + m)
};
constexpr PackTables pack_tables()
{
    PackTables t = {};
    for (uint32_t k = 0; k < 32; ++k)
        t.steps[k] = scale_step(4 * k) | scale_step(4 * k + 1) << 8 | scale_step(4 * k + 2) << 16 | scale_step(4 * k + 3) << 24;
    for (int m = 0; m < 8; ++m) t.inverses[m] = 8.0f * (1.0f - 0x1p-20f) / (float)(8 + m);
    return t;
}
static __device__ const PackTables kPackTables = pack_tables();
__device__ __forceinline__ int scale_byte(uint32_t amax, uint32_t table)               // by the whole warp
{
    const uint32_t m = amax & 127u, four = __shfl_sync(0xffffffffu, table, m >> 2);
    const int byte = 8 * ((int)(amax >> 7) - 110) + (int)((four >> (8 * (m & 3))) & 255u);
    return max(byte, 0);
}
__device__ __forceinline__ float scale_value(int byte) { return __uint_as_float(((uint32_t)byte << 20) + ((127u - kScaleBias) << 23)); }
// What a value is multiplied by: 1 / s, 2^-20 of it less.  Products are then below the exact quotient by 2^-21 to 2^-19 of it, so that
// a value halfway between two multiples of s goes to the smaller one; any other quotient is 2^-9 of itself from a halfway point.
// `table`: lane m holds that of (8 + m % 8) / 8.
__device__ __forceinline__ float scale_inverse(int byte, float table)                  // by the whole warp
{
    return __uint_as_float(__float_as_uint(__shfl_sync(0xffffffffu, table, byte & 7)) + (uint32_t)(kScaleBias - (byte >> 3)) * (1u << 23));
}
// The pattern of the float 12582912 + c, c = 8 + the nearest whole number to x / s (one rounding, of the exact x * inv + 12582920);
// |x| is at most kPackLargest or 7 17/16 s, so c is 1 .. 15.  The patterns' upper 16 bits vanish from sums of 16^k times them.
__device__ __forceinline__ uint32_t code_bits(float x, float inv) { return __float_as_uint(fmaf(x, inv, 12582920.0f)); }
// Four codes in the lower 16 bits.
__device__ __forceinline__ uint32_t code_half(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3) { return c0 + 16u * c1 + 256u * c2 + 4096u * c3; }

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

// The 4-bit form of a prefix cache: blocks of 32 values, e2m1 codes and one power-of-two scale each
// (layout and definition: mcsd.h).  gfx950 converts both ways by itself, two values an instruction,
// with the scale as the exponent of a float operand: rounding to nearest even, saturating at 6.
#pragma once

#include "mcsd_internal.h"

namespace mcsd {

constexpr int FB_BLOCK = 32;        // values per block
constexpr int FB_TILE = 16;         // rows per tile of the layout

// Where block `blk` of pool row `row` (rows of one (page, KV head) counted through the pool) lies, in blocks.  A tile
// holds its blocks column by column: the 16 blocks of the same columns are 256 bytes.
__device__ __forceinline__ size_t fourbit_block(size_t row, int n_blocks, int blk)
{
    return (row / FB_TILE * n_blocks + blk) * FB_TILE + row % FB_TILE;
}

// Scale byte of a block by the bits of its largest magnitude: with amax = 1.M 2^(E-127), 7 2^e >= amax
// means 1.M <= 1.75 at e = E - 129 and e = E - 128 otherwise.  Clamped so that every code value times the scale is
// a normal finite bf16.
__device__ __forceinline__ uint32_t fourbit_scale_byte(uint32_t amax_bits)
{
    const int E = (int)(amax_bits >> 23);
    if (E == 255) return 255u;
    return (uint32_t)min(max(E - ((amax_bits & 0x7fffffu) <= 0x600000u ? 2 : 1), 8), 252);
}

// The converters' scale operand: a float of which they use the exponent (s = 255, no number, makes every value NaN).
__device__ __forceinline__ float fourbit_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight values -> their codes, the first in the low bits.  A block that is not finite (s = 255) holds zeros.
__device__ __forceinline__ uint32_t fourbit_encode8(const float *x, uint32_t scale_byte)
{
    const float s = fourbit_scale(scale_byte);
    uint32_t c = 0u;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
    return scale_byte == 255u ? 0u : c;
}

// Four lanes hold a block, eight values each: bits of the largest magnitude of all 32.
__device__ __forceinline__ uint32_t fourbit_amax_bits(const float *x)
{
    // (magnitudes compare as their bits do, and anything that is not finite lies above all numbers)
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    return max(m, (uint32_t)__shfl_xor((int)m, 2));
}

// Eight values of a row in memory, 16-byte aligned.
__device__ __forceinline__ void load8(const char *at, bool is_f32, float *x)
{
    if (is_f32) {
        const float4 a = *reinterpret_cast<const float4 *>(at), b = *reinterpret_cast<const float4 *>(at + 16);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(at);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

}  // namespace mcsd

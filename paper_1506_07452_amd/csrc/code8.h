// Activations held in 8 bits (device side).  A flat tensor is cut into blocks
// of 64 consecutive elements; a block has one bf16 scale and an int8 code per
// element:
//   top   = max |x| over the block
//   scale = the smallest bf16 number >= top / 127
//   code  = x / scale to the nearest integer, ties to even    (|code| <= 127)
//   value = code * scale                                       (15 bits: exact)
// An error of half a scale, so at most top / 252 (bf16 has 8 bits: scale <=
// top / 127 (1 + 2^-7)).  A block whose top is below 2^-119 (where the scale
// would leave bf16's normal range) has scale 0 and codes 0.  A block with an
// infinity or a NaN has scale NaN: its values are NaN, so that a checkpoint
// never hides a divergence.
#pragma once

#include "common.h"

namespace plstm {

constexpr int kCodeBlock = 64;
constexpr uint32_t kCodeSmallBits = 0x04000000u;   // 2^-119
constexpr uint32_t kInfBits = 0x7f800000u;

inline long long code_blocks(long long n) { return (n + kCodeBlock - 1) / kCodeBlock; }

__device__ inline uint32_t float_bits(float f) { return __builtin_bit_cast(uint32_t, f); }
__device__ inline float bits_float(uint32_t u) { return __builtin_bit_cast(float, u); }

// Scale (bf16 bits) of a block from the bits of its largest magnitude, taken
// as integers so that a NaN is the largest of all.
__device__ inline uint16_t code_scale(uint32_t top_bits)
{
    if (top_bits >= kInfBits) return 0x7fc0u;
    if (top_bits < kCodeSmallBits) return 0;
    // top times 1/127 rounded is within two steps of fp32 of top / 127: cut to 8 bits it is the
    // scale or one or two below.  8-bit by 7-bit products are exact.
    const float top = bits_float(top_bits);
    uint32_t s = float_bits(top * (1.0f / 127.0f)) & 0xffff0000u;
    s += bits_float(s) * 127.0f < top ? 0x10000u : 0u;
    s += bits_float(s) * 127.0f < top ? 0x10000u : 0u;
    return (uint16_t)(s >> 16);
}

// Codes of a block with a scale, in the low byte of what code() gives.  Added to
// 3 2^22 a value is rounded to an integer, ties to even, whose two's complement is in
// the low bits; a block of zeros or NaNs has r = 0 and gets zeros (NaN: any byte is
// cleared by `keep`).
struct Coder {
    float s, half_s, r;             // r: 1 / s within an ulp
    uint32_t keep;
    __device__ explicit Coder(uint16_t scale)
    {
        const bool zero = scale == 0 || scale == 0x7fc0u;
        s = zero ? 0.0f : bf16_to_f32(scale);
        half_s = 0.5f * s;
        r = zero ? 0.0f : __builtin_amdgcn_rcpf(s);
        keep = zero ? 0u : ~0u;
    }
    // fp32 input: x r is within 1e-5 of x / s, so its nearest integer q is the
    // right one or, next to a tie, the one beside it.  The remainder x - q s
    // is exact in one fma (both operands are multiples of a bit that is at
    // most 2^-17 of s); past half a scale, or at half with q odd, the
    // neighbour on its side is taken.
    __device__ uint32_t code(float x) const
    {
        const float m = 12582912.0f;
        const float t = fmaf(x, r, m);
        const float rem = fmaf(m - t, s, x);
        const uint32_t c = float_bits(t), a = float_bits(rem) & 0x7fffffffu;
        return c + (a + (c & 1u) > float_bits(half_s) ? (rem > 0.0f ? 1u : ~0u) : 0u);
    }
    // bf16 input: x / s is a tie or at least 2^-9 from one (both have 8 bits),
    // and x r is within 2^-14 of it.  Added to 3 2^12 and taken away again it is
    // rounded to a multiple of 2^-10: ties come out as ties, nothing else does.
    __device__ uint32_t code_bf16(float x) const
    {
        const float k = 12288.0f;
        return float_bits((fmaf(x, r, k) - k) + 12582912.0f);
    }
};

}  // namespace plstm

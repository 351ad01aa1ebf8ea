// Rows in 4 bits: 128 channels in 80 bytes.  64 bytes of codes (channel 2 j in the low half of byte j, 2 j + 1 in the high half), then for
// each group of 32 channels two bf16, the step s and the least value lo.  A channel of code c stands for lo + s c.
//
//   s = (greatest - least) / 15 rounded up to four significant bits,  c = ceil((x - lo) / s - 1/2)
//
// With four significant bits in s and four in c the product s c is exact in bf16, so that it can enter a matrix instruction as it is; lo,
// a value of the row, is one as well.  The rounding up costs 5 % of the step on average (groups of 32 normal values).  A step below 2^-120 is 0 (all codes 0); a group
// that holds a value which is not finite, or whose step exceeds 2^120, is held as not a number throughout.
#pragma once
#include "two.cuh"

namespace compactor {

constexpr int kRow4 = 80;                      // bytes of a row
constexpr int kRow4Codes = 64;                 // the steps and least values begin here

__device__ __forceinline__ uint32_t min_nan2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
// Eight channels of a row in each lane, a group in four neighbouring lanes: the word of codes, and in `param` the group's s (lower half) and lo.
// All lanes of the warp call it.
__device__ __forceinline__ uint32_t quantise8(const uint4& x, uint32_t& param) {
    uint32_t least = min_nan2(min_nan2(x.x, x.y), min_nan2(x.z, x.w)), most = max_nan2(max_nan2(x.x, x.y), max_nan2(x.z, x.w));
#pragma unroll
    for (int d = 1; d <= 2; d *= 2) {
        least = min_nan2(least, __shfl_xor_sync(0xffffffffu, least, d));
        most = max_nan2(most, __shfl_xor_sync(0xffffffffu, most, d));
    }
    least = min_nan2(least, least >> 16 | least << 16);      // both halves the same
    most = max_nan2(most, most >> 16 | most << 16);
    const float lo = bf16_hi(least) + 0.f;                   // (-0 is 0)
    // The least number s of four significant bits with 15 s >= the range: rounded up from a quotient that is a little small, and one up if that was
    // too little (15 s is exact).
    const float range = bf16_hi(most) - lo;
    float s = __uint_as_float((__float_as_uint(range * ((1.f - 0x1p-22f) / 15.f)) + 0xfffffu) & ~0xfffffu);
    if (15.f * s < range) s = __uint_as_float(__float_as_uint(s) + 0x100000u);
    const bool good = range <= 15.f * 0x1p120f;              // (false for not a number)
    if (s < 0x1p-120f) s = 0.f;
    param = good ? __float_as_uint(s) >> 16 | __float_as_uint(lo) : 0x7fff7fffu;
    // The quotient by a reciprocal that is a little small gives the right code or, next to a border, the one below it: the remainder, which
    // is exact, tells.  (A division for each channel is twice the instructions, and this is what the fill spends most of them on.)
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    inv *= 1.f - 0x1p-21f;
    const float half = 0.5f * s;
    const uint32_t in[4] = {x.x, x.y, x.z, x.w};
    constexpr float kWhole = 12582912.f;                     // 1.5 2^23: added to it, a number is rounded to a whole one in its low bits
    uint32_t codes = 0;
#pragma unroll
    for (int j = 3; j >= 0; --j) {                           // two channels at a time
        const Two d = add_two(two(bf16_lo(in[j]), bf16_hi(in[j])), two(-lo, -lo));
        const Two t = fma_two(d, two(inv, inv), two(kWhole, kWhole));
        const Two rest = fma_two(two(-s, -s), add_two(t, two(-kWhole, -kWhole)), d);
        float t0, t1, r0, r1;
        split_two(t, t0, t1);
        split_two(rest, r0, r1);
        uint32_t even = __float_as_uint(t0), odd = __float_as_uint(t1);
        if (r0 > half) ++even;
        if (r1 > half) ++odd;
        codes = (codes * 16u + odd) * 16u + even;
    }
    return good && s > 0.f ? codes - 0x4b400000u * 0x11111111u : 0u;         // (without the eight bit patterns of 1.5 2^23)
}

// The eight values of a word of codes, rounded to bf16.
__device__ __forceinline__ uint4 values8(uint32_t codes, uint32_t param) {
    const float s = bf16_lo(param), lo = bf16_hi(param);
    uint32_t out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = __fmaf_rn(s, (float)((codes >> (8 * j)) & 15u), lo), b = __fmaf_rn(s, (float)((codes >> (8 * j + 4)) & 15u), lo);
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        out[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

}  // namespace compactor

// Microscaled 4-bit numbers: blocks of 32 e2m1 codes with one scale byte c, which stands for 2^(c - 127).
#pragma once
#include "sfs_common.cuh"

namespace sfs {
namespace mx4 {

constexpr int kCacheLo = 65, kCacheHi = 192;               // scales of a cache: value * 2^-64 is a normal bf16, or exact below it

#ifdef __CUDACC__
// The scale of a block from the bits of its largest magnitude (a NaN or an infinity has the largest bits of all).
__device__ __forceinline__ int scale_of(uint32_t amax_bits, int lo, int hi)
{
    if (amax_bits >= 0x7F800000u) return 255;
    return min(hi, max(lo, (int)(amax_bits >> 23) - 2));    // (below the normal numbers the exponent field is 0)
}
// 2^(127 - c): a normal number for every scale a finite block gets (c <= 252); 0 for the blocks that hold a NaN, whose codes are 0
__device__ __forceinline__ float inverse_scale(int c) { return c == 255 ? 0.f : __uint_as_float((uint32_t)(254 - c) << 23); }

// eight values -> eight codes, the first in the lowest nibble; to nearest, ties to even, saturated at 6
__device__ __forceinline__ uint32_t encode8(const float *y)
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
    return r;
}
// The two codes at bits 4 j of each half of `w` as bf16 times 2^-126: the sign goes to bit 15, the other three bits to the low end of the
// exponent and the high end of the mantissa, where 0.5 becomes a subnormal number of the right value.  One multiplication puts a copy at
// each place, a mask keeps the bits wanted: logic runs at half the rate of issue, and with two shifts instead of the multiplication (the
// other pipe's work) it was what bounded the decoding (single tokens of four sequences of 65536: 105 us).
template <int J>
__device__ __forceinline__ uint32_t codes_as_bf16(uint32_t w)
{
    const uint32_t x = J >= 2 ? w >> 8 : w;                 // (shared by both of its codes)
    return ((J & 1) ? (x & 0x00F000F0u) * 0x0104u : (x & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// A cache's scale as the one factor that turns codes_as_bf16 into values times 2^-64: 2^(c - 65), NaN above a cache's range.
__device__ __forceinline__ uint32_t cache_factor(uint32_t c) { return c > kCacheHi ? 0x7FC0u : (c + 62) << 7; }
// Eight codes -> eight values as bf16, in order.  2^(c - 1) goes in as two factors that are normal numbers for every c; every value is
// a bf16 number (the smallest, 2^-128, a subnormal one), so nothing is rounded.
__device__ __forceinline__ uint4 decode8(uint32_t w, uint32_t c)
{
    const uint32_t e = c + 126;                             // c - 1 = (e >> 1) + (e - (e >> 1)) - 127
    uint32_t f1 = ((e >> 1) + 63) << 7, f2 = (e - (e >> 1) + 64) << 7;
    if (c == 255) f1 = 0x7FC0u;
    f1 |= f1 << 16; f2 |= f2 << 16;
    const uint32_t h0 = mul_bf16x2(mul_bf16x2(codes_as_bf16<0>(w), f1), f2), h1 = mul_bf16x2(mul_bf16x2(codes_as_bf16<1>(w), f1), f2);
    const uint32_t h2 = mul_bf16x2(mul_bf16x2(codes_as_bf16<2>(w), f1), f2), h3 = mul_bf16x2(mul_bf16x2(codes_as_bf16<3>(w), f1), f2);
    return make_uint4(__byte_perm(h0, h1, 0x5410), __byte_perm(h2, h3, 0x5410), __byte_perm(h0, h1, 0x7632), __byte_perm(h2, h3, 0x7632));
}
#endif

}  // namespace mx4

// The current device's status word, allocated on first use, which a capture of `stream` does not allow (and would not survive).
int32_t status_word_outside_captures(cudaStream_t stream, int32_t **word);
}  // namespace sfs

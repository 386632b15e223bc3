// Microscaled 4-bit numbers: blocks of 32 e2m1 codes with one scale byte c, which stands for 2^(c - 127).
#pragma once
#include "sfs_common.cuh"
#include <cuda_fp16.h>

namespace sfs {
namespace mx4 {

constexpr int kBlock = 32;
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
// 2^(c - 127), NaN for 255
__device__ __forceinline__ float scale_value(int c) { return __uint_as_float(c == 0 ? 0x00400000u : c == 255 ? 0x7FC00000u : (uint32_t)c << 23); }

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
// The two codes at bits 4 j of each half of `w` as fp16 times 2^-14: sign to bit 15, the other three bits to the low end of the
// exponent and the high end of the mantissa, where 0.5 becomes a subnormal number of the right value.
template <int J>
__device__ __forceinline__ uint32_t codes_as_fp16(uint32_t w)
{
    const uint32_t s = J == 3 ? w : w << (12 - 4 * J);
    const uint32_t m = J == 0 ? w << 9 : J == 1 ? w << 5 : J == 2 ? w << 1 : w >> 3;
    return (s & 0x80008000u) | (m & 0x0E000E00u);
}
// eight codes -> eight values without their scale
__device__ __forceinline__ void decode8(uint32_t w, float *v)
{
    uint32_t h[4];
    h[0] = codes_as_fp16<0>(w); h[1] = codes_as_fp16<1>(w); h[2] = codes_as_fp16<2>(w); h[3] = codes_as_fp16<3>(w);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[j]));
        v[j] = f.x * 16384.f; v[j + 4] = f.y * 16384.f;
    }
}
#endif

}  // namespace mx4
}  // namespace sfs

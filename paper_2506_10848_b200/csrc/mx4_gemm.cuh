// The product of two matrices of microscaled 4-bit numbers: what its kernels share.
#pragma once
#include "mx4.cuh"

namespace sfs {

namespace mx4 {
constexpr int kDepth = 256;                                 // columns of a stage
constexpr int kCodes = 128;                                 // bytes of a row in a stage
constexpr int kScaleTile = 512;                             // 128 rows x 4 blocks

}  // namespace mx4

struct Mx4Args {
    const uint8_t *lane_scales, *col_scales;
    void *C; long long ldc;
    int lanes, cols;                                        // rows of the two operands
    int blocks, quads;                                      // blocks of 32 columns in a row, tiles of four of them
    int col_tiles, splits;
    int out_f32, features_on_lanes, wide, unit;             // wide: rows of C take 16-byte stores; unit: the widest that they all take
    float scale;
    int32_t *err;
};


namespace mx4 {
// kind::mxf4, both operands e2m1 and K-major, E8M0 scales of 32 columns, fp32 accumulator; `half`: which two of a column's four scale bytes
__host__ __device__ constexpr uint32_t idesc_mxf4(int M, int N, int half) { return ((uint32_t)(2 * half) << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 7) << 27) | ((uint32_t)(2 * half) << 29); }

#ifdef __CUDACC__
// shared-memory descriptor of 32 rows of 16 bytes, a scale tile as tcgen05.cp reads it: 8 rows are 128 consecutive bytes
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem) { return (uint64_t)((smem >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46); }
__device__ __forceinline__ void mma_mxf4_elect(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a, uint32_t scale_b, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred P, Q;\n\telect.sync _|P, 0xffffffff;\n\tsetp.ne.b32 Q, %6, 0;\n\t"
                 "@P tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], Q;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory");
}
// 32 rows of 16 bytes -> the same 32 lanes of all four quarters of tensor memory, four columns
__device__ __forceinline__ void copy_scales_elect(uint32_t tmem, uint32_t smem)
{
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\t"
                 "@P tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem), "l"(scale_desc(smem)) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t smem, const void *global, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem), "l"(global), "r"(bytes), "r"(bar) : "memory");
}
// eight bf16 values to an aligned place of which `n` belong to the row
__device__ __forceinline__ void put_bf16(__nv_bfloat16 *at, const uint4 &v, int n)
{
    if (n >= 8) { *reinterpret_cast<uint4 *>(at) = v; return; }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) at[i] = __ushort_as_bfloat16((unsigned short)((i & 1) ? w[i / 2] >> 16 : w[i / 2]));
}
#endif
}  // namespace mx4

struct Mx4Operands { const void *lanes, *cols; long long ld_lanes, ld_cols; };
// Many tiles, of 128 tokens (lanes) x 256 features: persistent CTAs.
int32_t linear_mx4_many(const Mx4Args &a, const Mx4Operands &x, cudaStream_t stream);
constexpr int kMx4ManyCols = 256;

}  // namespace sfs

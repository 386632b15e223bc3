// C = scale * A * B^T of two matrices of microscaled 4-bit numbers: one thread per element of C.
#include "mx4.cuh"

namespace sfs {
namespace {

__global__ void __launch_bounds__(256)
linear_mx4_elements(const uint8_t *A, long long lda, const uint8_t *As, const uint8_t *B, long long ldb, const uint8_t *Bs, void *C, long long ldc,
                    int M, int N, int blocks, int out_f32, float scale)
{
    pdl_wait();
    pdl_trigger();
    const int n = blockIdx.x * 16 + (threadIdx.x & 15), m = blockIdx.y * 16 + threadIdx.x / 16, quads = (blocks + 3) / 4;
    if (m >= M || n >= N) return;
    auto place = [&](int r, int b) { return ((size_t)(r >> 7) * quads + (b >> 2)) * 512 + (r & 31) * 16 + ((r & 127) >> 5) * 4 + (b & 3); };
    float sum = 0.f;
    for (int b = 0; b < blocks; ++b) {
        float part = 0.f;
        for (int w = 0; w < 4; ++w) {
            float x[8], y[8];
            mx4::decode8(*reinterpret_cast<const uint32_t *>(A + m * lda + b * 16 + w * 4), x);
            mx4::decode8(*reinterpret_cast<const uint32_t *>(B + n * ldb + b * 16 + w * 4), y);
            for (int i = 0; i < 8; ++i) part = fmaf(x[i], y[i], part);
        }
        sum += part * mx4::scale_value(As[place(m, b)]) * mx4::scale_value(Bs[place(n, b)]);
    }
    sum *= scale;
    if (out_f32) static_cast<float *>(C)[m * ldc + n] = sum;
    else static_cast<__nv_bfloat16 *>(C)[m * ldc + n] = __float2bfloat16_rn(sum);
}

}  // namespace
}  // namespace sfs

using namespace sfs;

extern "C" int32_t sfs_linear_mx4(const void *d_A, int64_t lda, const void *d_A_scales, const void *d_B, int64_t ldb, const void *d_B_scales,
                                  void *d_C, int64_t ldc, int32_t M, int32_t N, int32_t K, int32_t out_dtype, float scale, void *stream)
{
    SFS_REQUIRE(d_A && d_B && d_C && d_A_scales && d_B_scales, SFS_ERR_INVALID_ARG, "linear_mx4: NULL pointer");
    SFS_REQUIRE(M >= 1 && N >= 1 && K >= 1, SFS_ERR_INVALID_ARG, "linear_mx4: M, N, K must be positive");
    SFS_REQUIRE(M <= (1 << 30) && N <= (1 << 30) && K <= (1 << 30), SFS_ERR_UNSUPPORTED, "linear_mx4: M, N or K above 2^30");
    SFS_REQUIRE(out_dtype == 0 || out_dtype == 1, SFS_ERR_INVALID_ARG, "linear_mx4: out_dtype %d", out_dtype);
    SFS_REQUIRE(aligned_to(d_A, 16) && aligned_to(d_B, 16) && aligned_to(d_A_scales, 16) && aligned_to(d_B_scales, 16), SFS_ERR_INVALID_ARG,
                "linear_mx4: codes and scales must be 16-byte aligned");
    const int64_t bytes = SFS_MX4_CODE_BYTES(K);
    SFS_REQUIRE(lda % 16 == 0 && ldb % 16 == 0 && lda >= bytes && ldb >= bytes, SFS_ERR_INVALID_ARG,
                "linear_mx4: lda and ldb must be multiples of 16 and hold a row");
    SFS_REQUIRE(ldc >= N && aligned_to(d_C, out_dtype ? 4 : 2), SFS_ERR_INVALID_ARG, "linear_mx4: misaligned C, or ldc below N");
    SFS_CUDA(launch_pdl(linear_mx4_elements, dim3((unsigned)((N + 15) / 16), (unsigned)((M + 15) / 16)), dim3(256), 0, (cudaStream_t)stream,
                        (const uint8_t *)d_A, (long long)lda, (const uint8_t *)d_A_scales, (const uint8_t *)d_B, (long long)ldb, (const uint8_t *)d_B_scales,
                        d_C, (long long)ldc, M, N, (K + 31) / 32, out_dtype, scale));
    return SFS_OK;
}

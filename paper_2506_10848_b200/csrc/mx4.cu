// Quantisation of matrices and of a key / value cache to microscaled 4-bit numbers, and the values they stand for.
//
// A half-warp takes 128 consecutive values of a row, four blocks of 32: a lane holds 8 of them (16 bytes of bf16), a block's
// largest magnitude is the maximum of the bit patterns over 4 lanes, so a NaN or an infinity shows in it, and each value is
// scaled by a power of two (exact) and rounded once, by the conversion instruction.  Everything moves once: bound by HBM.
#include "attention_cache4.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = kThreads / 16;                       // half-warps of a CTA

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// eight values of a row from column `col` on, zeros behind the last column
template <typename T>
__device__ __forceinline__ void load8(const T *row, int col, int cols, bool wide, float *v)
{
    if (wide && col + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = *reinterpret_cast<const float4 *>(row + col), b = *reinterpret_cast<const float4 *>(row + col + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(row + col);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_bits_to_f32(w[i] & 0xFFFFu); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < cols ? to_f32<T>(row[col + i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *row, int col, int cols, bool wide, const float *v)
{
    if (wide && col + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(row + col) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(row + col + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t *>(&h); }
            *reinterpret_cast<uint4 *>(row + col) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = from_f32<T>(v[i]);
    }
}

// the four lanes of a block: its scale, and this lane's eight codes
__device__ __forceinline__ uint32_t quantize8(float *v, int lo, int hi, int &c)
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
    c = mx4::scale_of(a, lo, hi);
    const float f = mx4::inverse_scale(c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= f;
    return c == 255 ? 0u : mx4::encode8(v);
}
__device__ __forceinline__ void dequantize8(uint32_t codes, int c, float *v)
{
    mx4::decode8(codes, v);
    const float f = mx4::scale_value(c);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= f;
}

// where the four scale bytes of a row's blocks 4 q .. 4 q + 3 lie in a matrix's tiles
__device__ __forceinline__ size_t scale_quad(int row, int q, int quads) { return ((size_t)(row >> 7) * quads + q) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4; }

// A half-warp's position, four blocks of a row, and the step to its next one without a division.
struct Walk {
    int row, quad, step_rows, step_quads, quads;
    __device__ __forceinline__ Walk(long long first, int stride, int quads_) : quads(quads_)
    {
        row = (int)(first / quads); quad = (int)(first - (long long)row * quads);
        step_rows = stride / quads; step_quads = stride - step_rows * quads;
    }
    __device__ __forceinline__ void next() { row += step_rows; quad += step_quads; if (quad >= quads) { quad -= quads; ++row; } }
};

template <typename T>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const T *__restrict__ x, long long ldx, int rows, int cols, uint8_t *__restrict__ codes, long long ld_codes,
                uint8_t *__restrict__ scales, int quads, int wide)
{
    pdl_wait();
    pdl_trigger();
    const int l = threadIdx.x & 15, blocks = (cols + 31) / 32, tile_rows = (rows + 127) / 128 * 128;
    Walk at((long long)blockIdx.x * kUnits + threadIdx.x / 16, gridDim.x * kUnits, quads);
    // (both halves of a warp run as long as either has work: the shuffles are the whole warp's)
    while (__any_sync(0xffffffffu, at.row < tile_rows)) {
        const int col = at.quad * 128 + l * 8;
        float v[8];
        if (at.row < rows) load8<T>(x + at.row * ldx, col, cols, wide != 0, v);
        else { for (int i = 0; i < 8; ++i) v[i] = 0.f; }
        int c;
        const uint32_t word = quantize8(v, 0, 254, c);
        const bool block_in = at.row < rows && at.quad * 4 + (l >> 2) < blocks;
        if (block_in) *reinterpret_cast<uint32_t *>(codes + at.row * ld_codes + at.quad * 64 + l * 4) = word;
        uint32_t s = (block_in ? (uint32_t)c : 0u) << ((l >> 2) * 8);         // the padding of the tiles holds zeros
        s |= __shfl_xor_sync(0xffffffffu, s, 4);
        s |= __shfl_xor_sync(0xffffffffu, s, 8);
        if (l == 0 && at.row < tile_rows) *reinterpret_cast<uint32_t *>(scales + scale_quad(at.row, at.quad, quads)) = s;
        at.next();
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t *__restrict__ codes, long long ld_codes, const uint8_t *__restrict__ scales, int rows, int cols, T *__restrict__ x,
                  long long ldx, int quads, int wide)
{
    pdl_wait();
    pdl_trigger();
    const int l = threadIdx.x & 15, blocks = (cols + 31) / 32;
    Walk at((long long)blockIdx.x * kUnits + threadIdx.x / 16, gridDim.x * kUnits, quads);
    while (at.row < rows) {
        const int b = at.quad * 4 + (l >> 2);
        if (b < blocks) {
            float v[8];
            dequantize8(*reinterpret_cast<const uint32_t *>(codes + at.row * ld_codes + at.quad * 64 + l * 4),
                        scales[scale_quad(at.row, at.quad, quads) + (l >> 2)], v);
            store8<T>(x + at.row * ldx, at.quad * 128 + l * 8, cols, wide != 0, v);
        }
        at.next();
    }
}

// ---- the cache: a token's keys (or values) of all heads are one row of blocks, codes and scales each in one run of bytes ------------

constexpr int kStoreRows = 8;                               // tokens of a CTA

template <typename T>
__global__ void __launch_bounds__(kThreads)
cache_store_kernel(uint8_t *__restrict__ k_codes, uint8_t *__restrict__ k_scales, uint8_t *__restrict__ v_codes, uint8_t *__restrict__ v_scales,
                   int n_slots, int width, const T *__restrict__ k, long long ld_k, const T *__restrict__ v, long long ld_v, int wide_k, int wide_v,
                   const int32_t *__restrict__ slots, int n_rows)
{
    pdl_wait();
    pdl_trigger();
    __shared__ int s_slot[kStoreRows];
    const int r0 = blockIdx.x * kStoreRows;
    if (threadIdx.x < kStoreRows) {
        const int r = r0 + threadIdx.x;
        const int slot = r < n_rows ? (slots ? slots[r] : r) : -1;
        s_slot[threadIdx.x] = (unsigned)slot < (unsigned)n_slots ? slot : -1;
    }
    __syncthreads();
    if (slots) {                                            // a later row with the same slot is the one that counts
        int mine[kStoreRows];
#pragma unroll
        for (int i = 0; i < kStoreRows; ++i) mine[i] = s_slot[i];
        __syncthreads();
        for (int r = r0 + 1 + threadIdx.x; r < n_rows; r += kThreads) {
            const int other = slots[r];
#pragma unroll
            for (int i = 0; i < kStoreRows; ++i)
                if (other == mine[i] && r > r0 + i) s_slot[i] = -1;
        }
        __syncthreads();
    }
    const bool keys = blockIdx.y == 0;
    const T *src = keys ? k : v;
    const long long ld = keys ? ld_k : ld_v;
    const bool wide = keys ? wide_k : wide_v;
    uint8_t *codes = keys ? k_codes : v_codes, *scales = keys ? k_scales : v_scales;
    const int blocks = width / 32, quads = (blocks + 3) / 4, l = threadIdx.x & 15;
    Walk at(threadIdx.x / 16, kUnits, quads);
    while (__any_sync(0xffffffffu, at.row < kStoreRows)) {
        const int slot = at.row < kStoreRows ? s_slot[at.row] : -1, b = at.quad * 4 + (l >> 2);
        const bool in = slot >= 0 && b < blocks;
        float x[8];
        if (in) load8<T>(src + (r0 + at.row) * ld, at.quad * 128 + l * 8, width, wide, x);
        else { for (int i = 0; i < 8; ++i) x[i] = 0.f; }
        int c;
        const uint32_t word = quantize8(x, mx4::kCacheLo, mx4::kCacheHi, c);
        if (in) {
            *reinterpret_cast<uint32_t *>(codes + (size_t)slot * (width / 2) + at.quad * 64 + l * 4) = word;
            if ((l & 3) == 0) scales[(size_t)slot * blocks + b] = (uint8_t)c;
        }
        at.next();
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
cache_load_kernel(const uint8_t *__restrict__ k_codes, const uint8_t *__restrict__ k_scales, const uint8_t *__restrict__ v_codes,
                  const uint8_t *__restrict__ v_scales, int n_slots, int width, T *__restrict__ k, long long ld_k, T *__restrict__ v, long long ld_v,
                  int wide_k, int wide_v, const int32_t *__restrict__ slots, int n_rows)
{
    pdl_wait();
    pdl_trigger();
    const bool keys = blockIdx.y == 0;
    T *dst = keys ? k : v;
    if (dst == nullptr) return;
    const long long ld = keys ? ld_k : ld_v;
    const bool wide = keys ? wide_k : wide_v;
    const uint8_t *codes = keys ? k_codes : v_codes, *scales = keys ? k_scales : v_scales;
    const int blocks = width / 32, quads = (blocks + 3) / 4, l = threadIdx.x & 15;
    Walk at((long long)blockIdx.x * kUnits + threadIdx.x / 16, gridDim.x * kUnits, quads);
    while (at.row < n_rows) {
        const int slot = slots ? slots[at.row] : at.row, b = at.quad * 4 + (l >> 2);
        if ((unsigned)slot < (unsigned)n_slots && b < blocks) {
            float x[8];
            const int c = scales[(size_t)slot * blocks + b];
            dequantize8(*reinterpret_cast<const uint32_t *>(codes + (size_t)slot * (width / 2) + at.quad * 64 + l * 4), c > mx4::kCacheHi ? 255 : c, x);
            store8<T>(dst + at.row * ld, at.quad * 128 + l * 8, width, wide, x);
        }
        at.next();
    }
}

bool wide_rows(const void *base, int64_t ld, size_t element) { return aligned_to(base, 16) && (ld * (int64_t)element) % 16 == 0; }
// CTAs for `units` half-warps of work: up to eight on an SM, at least a few units each
unsigned grid_for(long long units) { return (unsigned)std::max<long long>(1, std::min<long long>((units + kUnits - 1) / kUnits, (long long)gemm_num_sms() * 8)); }

}  // namespace

int32_t cache4_check(const sfs_cache4 *c, const char *what)
{
    SFS_REQUIRE(c && c->k_codes && c->k_scales && c->v_codes && c->v_scales, SFS_ERR_INVALID_ARG, "%s: NULL cache", what);
    SFS_REQUIRE(aligned_to(c->k_codes, 16) && aligned_to(c->k_scales, 16) && aligned_to(c->v_codes, 16) && aligned_to(c->v_scales, 16),
                SFS_ERR_INVALID_ARG, "%s: codes and scales must be 16-byte aligned", what);
    SFS_REQUIRE(c->batch >= 1 && c->capacity >= 1 && c->n_kv_heads >= 1, SFS_ERR_INVALID_ARG, "%s: bad cache sizes", what);
    SFS_REQUIRE((int64_t)c->batch * c->capacity <= 0x7FFFFFFF, SFS_ERR_INVALID_ARG, "%s: more slots than an int32 names", what);
    SFS_REQUIRE(c->head_dim == 64 || c->head_dim == 128, SFS_ERR_UNSUPPORTED, "%s: head_dim %d (64 or 128)", what, c->head_dim);
    SFS_REQUIRE(c->n_kv_heads <= 1024, SFS_ERR_UNSUPPORTED, "%s: more than 1024 key heads", what);
    return SFS_OK;
}

}  // namespace sfs

using namespace sfs;

static int32_t check_matrix(const char *what, const void *d_x, int64_t ldx, int32_t dtype, int32_t rows, int32_t cols, const void *d_codes,
                            int64_t ld_codes, const void *d_scales)
{
    SFS_REQUIRE(d_x && d_codes && d_scales, SFS_ERR_INVALID_ARG, "%s: NULL pointer", what);
    SFS_REQUIRE(rows >= 1 && cols >= 1, SFS_ERR_INVALID_ARG, "%s: rows and cols must be positive", what);
    SFS_REQUIRE(rows <= (1 << 30) && cols <= (1 << 30), SFS_ERR_UNSUPPORTED, "%s: rows or cols above 2^30", what);
    SFS_REQUIRE(dtype == SFS_LOGITS_BF16 || dtype == SFS_LOGITS_F32, SFS_ERR_INVALID_ARG, "%s: type %d", what, dtype);
    SFS_REQUIRE(ldx >= cols, SFS_ERR_INVALID_ARG, "%s: ldx below cols", what);
    SFS_REQUIRE(aligned_to(d_x, dtype == SFS_LOGITS_BF16 ? 2 : 4), SFS_ERR_INVALID_ARG, "%s: misaligned matrix", what);
    SFS_REQUIRE(aligned_to(d_codes, 16) && aligned_to(d_scales, 16), SFS_ERR_INVALID_ARG, "%s: codes and scales must be 16-byte aligned", what);
    SFS_REQUIRE(ld_codes % 16 == 0 && ld_codes >= SFS_MX4_CODE_BYTES(cols), SFS_ERR_INVALID_ARG, "%s: ld_codes must be a multiple of 16 and hold a row", what);
    return SFS_OK;
}

static int32_t check_rows(const char *what, const sfs_cache4 *c, const void *d, int64_t ld, int32_t dtype)
{
    SFS_REQUIRE(ld >= (int64_t)c->n_kv_heads * c->head_dim, SFS_ERR_INVALID_ARG, "%s: rows overlap", what);
    SFS_REQUIRE(aligned_to(d, dtype == SFS_LOGITS_BF16 ? 2 : 4), SFS_ERR_INVALID_ARG, "%s: misaligned rows", what);
    return SFS_OK;
}

extern "C" {

int32_t sfs_mx4_quantize(const void *d_x, int64_t ldx, int32_t in_dtype, int32_t rows, int32_t cols, void *d_codes, int64_t ld_codes,
                         void *d_scales, void *stream)
{
    const int32_t rc = check_matrix("mx4_quantize", d_x, ldx, in_dtype, rows, cols, d_codes, ld_codes, d_scales);
    if (rc != SFS_OK) return rc;
    const int quads = (cols + 127) / 128;
    const unsigned grid = grid_for((long long)((rows + 127) / 128 * 128) * quads);
    const size_t element = in_dtype == SFS_LOGITS_BF16 ? 2 : 4;
    const int wide = wide_rows(d_x, ldx, element);
    if (in_dtype == SFS_LOGITS_BF16)
        SFS_CUDA(launch_pdl(quantize_kernel<__nv_bfloat16>, dim3(grid), dim3(kThreads), 0, (cudaStream_t)stream, (const __nv_bfloat16 *)d_x, (long long)ldx,
                            rows, cols, (uint8_t *)d_codes, (long long)ld_codes, (uint8_t *)d_scales, quads, wide));
    else
        SFS_CUDA(launch_pdl(quantize_kernel<float>, dim3(grid), dim3(kThreads), 0, (cudaStream_t)stream, (const float *)d_x, (long long)ldx,
                            rows, cols, (uint8_t *)d_codes, (long long)ld_codes, (uint8_t *)d_scales, quads, wide));
    return SFS_OK;
}

int32_t sfs_mx4_dequantize(const void *d_codes, int64_t ld_codes, const void *d_scales, int32_t rows, int32_t cols, void *d_x, int64_t ldx,
                           int32_t out_dtype, void *stream)
{
    const int32_t rc = check_matrix("mx4_dequantize", d_x, ldx, out_dtype, rows, cols, d_codes, ld_codes, d_scales);
    if (rc != SFS_OK) return rc;
    const int quads = (cols + 127) / 128;
    const unsigned grid = grid_for((long long)rows * quads);
    const size_t element = out_dtype == SFS_LOGITS_BF16 ? 2 : 4;
    const int wide = wide_rows(d_x, ldx, element);
    if (out_dtype == SFS_LOGITS_BF16)
        SFS_CUDA(launch_pdl(dequantize_kernel<__nv_bfloat16>, dim3(grid), dim3(kThreads), 0, (cudaStream_t)stream, (const uint8_t *)d_codes, (long long)ld_codes,
                            (const uint8_t *)d_scales, rows, cols, (__nv_bfloat16 *)d_x, (long long)ldx, quads, wide));
    else
        SFS_CUDA(launch_pdl(dequantize_kernel<float>, dim3(grid), dim3(kThreads), 0, (cudaStream_t)stream, (const uint8_t *)d_codes, (long long)ld_codes,
                            (const uint8_t *)d_scales, rows, cols, (float *)d_x, (long long)ldx, quads, wide));
    return SFS_OK;
}

int32_t sfs_cache4_store(const sfs_cache4 *cache, const void *d_k, int64_t ld_k, const void *d_v, int64_t ld_v, int32_t in_dtype,
                         const int32_t *d_slots, int32_t n_rows, void *stream)
{
    int32_t rc = cache4_check(cache, "cache4_store");
    if (rc != SFS_OK) return rc;
    SFS_REQUIRE(d_k && d_v, SFS_ERR_INVALID_ARG, "cache4_store: NULL pointer");
    SFS_REQUIRE(in_dtype == SFS_LOGITS_BF16 || in_dtype == SFS_LOGITS_F32, SFS_ERR_INVALID_ARG, "cache4_store: type %d", in_dtype);
    SFS_REQUIRE(n_rows >= 0, SFS_ERR_INVALID_ARG, "cache4_store: n_rows %d", n_rows);
    SFS_REQUIRE(aligned_to(d_slots, 4), SFS_ERR_INVALID_ARG, "cache4_store: misaligned slots");
    if ((rc = check_rows("cache4_store", cache, d_k, ld_k, in_dtype)) != SFS_OK || (rc = check_rows("cache4_store", cache, d_v, ld_v, in_dtype)) != SFS_OK) return rc;
    if (n_rows == 0) return SFS_OK;
    const int n_slots = cache->batch * cache->capacity, width = cache->n_kv_heads * cache->head_dim;
    const size_t element = in_dtype == SFS_LOGITS_BF16 ? 2 : 4;
    const int wk = wide_rows(d_k, ld_k, element), wv = wide_rows(d_v, ld_v, element);
    const dim3 grid((unsigned)((n_rows + kStoreRows - 1) / kStoreRows), 2);
    uint8_t *kc = (uint8_t *)cache->k_codes, *ks = (uint8_t *)cache->k_scales, *vc = (uint8_t *)cache->v_codes, *vs = (uint8_t *)cache->v_scales;
    if (in_dtype == SFS_LOGITS_BF16)
        SFS_CUDA(launch_pdl(cache_store_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, (cudaStream_t)stream, kc, ks, vc, vs, n_slots, width,
                            (const __nv_bfloat16 *)d_k, (long long)ld_k, (const __nv_bfloat16 *)d_v, (long long)ld_v, wk, wv, d_slots, n_rows));
    else
        SFS_CUDA(launch_pdl(cache_store_kernel<float>, grid, dim3(kThreads), 0, (cudaStream_t)stream, kc, ks, vc, vs, n_slots, width,
                            (const float *)d_k, (long long)ld_k, (const float *)d_v, (long long)ld_v, wk, wv, d_slots, n_rows));
    return SFS_OK;
}

int32_t sfs_cache4_load(const sfs_cache4 *cache, const int32_t *d_slots, int32_t n_rows, void *d_k, int64_t ld_k, void *d_v, int64_t ld_v,
                        int32_t out_dtype, void *stream)
{
    int32_t rc = cache4_check(cache, "cache4_load");
    if (rc != SFS_OK) return rc;
    SFS_REQUIRE(out_dtype == SFS_LOGITS_BF16 || out_dtype == SFS_LOGITS_F32, SFS_ERR_INVALID_ARG, "cache4_load: type %d", out_dtype);
    SFS_REQUIRE(n_rows >= 0, SFS_ERR_INVALID_ARG, "cache4_load: n_rows %d", n_rows);
    SFS_REQUIRE(aligned_to(d_slots, 4), SFS_ERR_INVALID_ARG, "cache4_load: misaligned slots");
    if (d_k && (rc = check_rows("cache4_load", cache, d_k, ld_k, out_dtype)) != SFS_OK) return rc;
    if (d_v && (rc = check_rows("cache4_load", cache, d_v, ld_v, out_dtype)) != SFS_OK) return rc;
    if (n_rows == 0 || (!d_k && !d_v)) return SFS_OK;
    const int n_slots = cache->batch * cache->capacity, width = cache->n_kv_heads * cache->head_dim;
    const size_t element = out_dtype == SFS_LOGITS_BF16 ? 2 : 4;
    const int wk = wide_rows(d_k, ld_k, element), wv = wide_rows(d_v, ld_v, element);
    const dim3 grid(grid_for((long long)n_rows * ((width + 127) / 128)), 2);
    const uint8_t *kc = (const uint8_t *)cache->k_codes, *ks = (const uint8_t *)cache->k_scales;
    const uint8_t *vc = (const uint8_t *)cache->v_codes, *vs = (const uint8_t *)cache->v_scales;
    if (out_dtype == SFS_LOGITS_BF16)
        SFS_CUDA(launch_pdl(cache_load_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, (cudaStream_t)stream, kc, ks, vc, vs, n_slots, width,
                            (__nv_bfloat16 *)d_k, (long long)ld_k, (__nv_bfloat16 *)d_v, (long long)ld_v, wk, wv, d_slots, n_rows));
    else
        SFS_CUDA(launch_pdl(cache_load_kernel<float>, grid, dim3(kThreads), 0, (cudaStream_t)stream, kc, ks, vc, vs, n_slots, width,
                            (float *)d_k, (long long)ld_k, (float *)d_v, (long long)ld_v, wk, wv, d_slots, n_rows));
    return SFS_OK;
}

}  // extern "C"

// Attention over a key / value cache of microscaled 4-bit numbers: one warp per query row and head.
#include "attention_cache4.cuh"

namespace sfs {
namespace {

template <int DH>
__global__ void __launch_bounds__(128)
attention_cache4_rows(Cache4Args a)
{
    pdl_wait();
    pdl_trigger();
    constexpr int E = DH / 32;                              // dimensions of a lane
    const int lane = threadIdx.x & 31, heads = a.n_kv * a.group;
    const long long item = (long long)blockIdx.x * 4 + threadIdx.x / 32;
    if (item >= (long long)a.batch * a.n_q * heads) return;
    const int head = (int)(item % heads), kv = head / a.group;
    const long long row = item / heads;
    const int b = (int)(row / a.n_q), i = (int)(row % a.n_q), length = cache4_length(a, b);
    long long p = (long long)length - a.n_q + i;
    if (a.positions) { p = a.positions[row]; if (p < 0) return; }
    const Seen seen = cache4_seen(a, length, p);
    float q[E], o[E], m = -INFINITY, l = 0.f;
    for (int e = 0; e < E; ++e) { q[e] = __bfloat162float(a.q[row * a.ld_q + head * DH + lane * E + e]); o[e] = 0.f; }
    auto value = [&](const uint8_t *codes, const uint8_t *scales, size_t at, float *v) {
        const int c = scales[at * (DH / 32) + lane * E / 32];
        const float f = mx4::scale_value(c > mx4::kCacheHi ? 255 : c);
        for (int e = 0; e < E; e += 2) {
            const uint32_t w = codes[at * (DH / 2) + (lane * E + e) / 2];
            float d[8];
            mx4::decode8(w, d);
            v[e] = d[0] * f; v[e + 1] = d[1] * f;
        }
    };
    for (int j = 0; j < seen.hi; ++j) {
        if (j >= seen.first && j < seen.lo) { j = seen.lo - 1; continue; }
        const size_t at = ((size_t)b * a.capacity + j) * a.n_kv + kv;
        float k[E], v[E], s = 0.f;
        value(a.k_codes, a.k_scales, at, k);
        value(a.v_codes, a.v_scales, at, v);
        for (int e = 0; e < E; ++e) s = fmaf(q[e], k[e], s);
        s = warp_sum(s) * a.scale_log2;
        const float m1 = fmaxf(m, s), base = m1 == -INFINITY ? 0.f : m1, f = exp2f(m - base), w = exp2f(s - base);
        l = l * f + w;
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * v[e];
        m = m1;
    }
    for (int e = 0; e < E; ++e) a.out[row * a.ld_out + head * DH + lane * E + e] = __float2bfloat16_rn(l == 0.f ? 0.f : o[e] / l);
}

}  // namespace
}  // namespace sfs

using namespace sfs;

extern "C" int32_t sfs_attention_cache4(const sfs_cache4 *cache, const void *d_q, int64_t ld_q, void *d_out, int64_t ld_out, int32_t n_heads,
                                        int32_t n_q, const int32_t *d_lengths, const int32_t *d_positions, int32_t left, int32_t right,
                                        int32_t sinks, void *stream)
{
    const int32_t rc = cache4_check(cache, "attention_cache4");
    if (rc != SFS_OK) return rc;
    SFS_REQUIRE(d_q && d_out, SFS_ERR_INVALID_ARG, "attention_cache4: NULL pointer");
    SFS_REQUIRE(n_heads >= 1 && n_heads % cache->n_kv_heads == 0, SFS_ERR_INVALID_ARG, "attention_cache4: n_heads must be a multiple of n_kv_heads");
    SFS_REQUIRE(n_heads <= 65535, SFS_ERR_UNSUPPORTED, "attention_cache4: more than 65535 heads");
    SFS_REQUIRE(n_q >= 0 && sinks >= 0, SFS_ERR_INVALID_ARG, "attention_cache4: n_q and sinks must not be negative");
    SFS_REQUIRE((int64_t)cache->batch * n_q <= 0x7FFFFFFF, SFS_ERR_INVALID_ARG, "attention_cache4: more rows than an int32 names");
    const int64_t width = (int64_t)n_heads * cache->head_dim;
    SFS_REQUIRE(ld_q >= width && ld_out >= width, SFS_ERR_INVALID_ARG, "attention_cache4: rows overlap");
    SFS_REQUIRE(aligned_to(d_q, 16) && aligned_to(d_out, 16) && ld_q % 8 == 0 && ld_out % 8 == 0, SFS_ERR_INVALID_ARG,
                "attention_cache4: queries and outputs must be 16-byte aligned, row by row");
    SFS_REQUIRE(aligned_to(d_lengths, 4) && aligned_to(d_positions, 4), SFS_ERR_INVALID_ARG, "attention_cache4: misaligned lengths or positions");
    if (n_q == 0) return SFS_OK;
    Cache4Args a = {(const uint8_t *)cache->k_codes, (const uint8_t *)cache->k_scales, (const uint8_t *)cache->v_codes, (const uint8_t *)cache->v_scales,
                    cache->batch, cache->capacity, cache->n_kv_heads, n_heads / cache->n_kv_heads,
                    (const __nv_bfloat16 *)d_q, (long long)ld_q, (__nv_bfloat16 *)d_out, (long long)ld_out, n_q, d_lengths, d_positions,
                    left, right, sinks, (float)(1.4426950408889634 / sqrt((double)cache->head_dim)), nullptr};
    const long long items = (long long)cache->batch * n_q * n_heads;
    SFS_REQUIRE(items / 4 < 0x7FFFFFFF, SFS_ERR_UNSUPPORTED, "attention_cache4: too many rows and heads for one call");
    SFS_CUDA(launch_pdl(cache->head_dim == 128 ? attention_cache4_rows<128> : attention_cache4_rows<64>, dim3((unsigned)((items + 3) / 4)), dim3(128), 0,
                        (cudaStream_t)stream, a));
    return SFS_OK;
}

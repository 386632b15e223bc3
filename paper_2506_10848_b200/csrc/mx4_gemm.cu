// C = scale * A * B^T of two matrices of microscaled 4-bit numbers on the block-scaled tensor-core instruction
// (tcgen05.mma kind::mxf4: 64 columns per step, two scale bytes per row and step read from tensor memory).
//
// A CTA computes a tile of 128 rows of one operand ("lanes") by BN rows of the other ("columns"): with many tokens the lanes are
// tokens, with at most 128 of them the lanes are features, so that one column tile of 16 .. 128 holds all tokens and the weights
// stream through every SM.  A stage of the shared-memory ring is 256 columns of codes (128 bytes a row, 128-byte swizzle, by TMA) and
// the scale tiles that belong to them, which lie in global memory as the copy into tensor memory wants them: 512 bytes for 128
// rows and 128 columns, one bulk copy.  Warp 0 loads, warp 1 copies scales to tensor memory and issues (both in the order of issue on
// the tensor core's pipe), warps 2-5 store.
//
// Few tiles: K is divided over a cluster of up to 8 CTAs, whose 32-bit partial sums are exchanged through shared memory and added
// in the order of the ranks, so no workspace and no atomics are needed and the same call gives the same bits.
#include "mx4_gemm.cuh"
#include "tc05.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

constexpr int kThreads = 192;
using namespace mx4;

template <int BN> struct Shape {
    static constexpr int kRowTiles = BN > 128 ? 2 : 1;      // scale tiles along the columns' rows (a tile of 192 starts in the middle of one, or ends there)
    static constexpr int kA = 128 * kCodes, kB = BN * kCodes;
    static constexpr int kScaleA = 2 * kScaleTile, kScaleB = kRowTiles * 2 * kScaleTile;
    static constexpr int kStage = kA + kB + kScaleA + kScaleB;
    static constexpr int kScaleCols = 8 + 8 * kRowTiles;    // tensor-memory columns of a stage's scales
    // stages of the ring with one or two CTAs on an SM: a lone CTA needs twice as many, or the memory's latency sets its pace
    static constexpr int stages(int per_sm) { return (per_sm == 1 ? 210 * 1024 : 106 * 1024) / kStage; }
    // every stage has scales of its own in tensor memory: a copy may overtake an MMA issued before it, but not the stage's release
    static constexpr uint32_t tmem_columns(int stages) { const int n = BN + stages * kScaleCols; return n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512; }
    static constexpr int shared(int stages) { return stages * kStage + 1024 /* alignment */ + (2 * stages + 1) * 8 + 16; }
    static_assert(kB % 1024 == 0 && BN + stages(1) * kScaleCols <= 512 && 2 * tmem_columns(stages(2)) <= 512 + (BN > 128 ? 512 : 0), "tile");
    static_assert(2 * kStage >= 128 * BN * 4 || BN > 128, "partial sums fit the ring");
};

__device__ __forceinline__ float load_remote(uint32_t cluster_addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
    return v;
}

// n consecutive columns of one lane
template <int N>
__device__ __forceinline__ void store_columns(const Mx4Args &a, int lane, int col, const float *v)
{
    if (lane >= a.lanes) return;
    if (a.features_on_lanes) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (col + i < a.cols) {
                const long long at = (long long)(col + i) * a.ldc + lane;
                if (a.out_f32) static_cast<float *>(a.C)[at] = v[i]; else static_cast<__nv_bfloat16 *>(a.C)[at] = __float2bfloat16_rn(v[i]);
            }
    } else {
        const long long at = (long long)lane * a.ldc + col;
        if (a.wide && N % 8 == 0 && !a.out_f32) {
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) { const __nv_bfloat162 h = __floats2bfloat162_rn(v[8 * i + 2 * t], v[8 * i + 2 * t + 1]); w[t] = *reinterpret_cast<const uint32_t *>(&h); }
                put_bf16(static_cast<__nv_bfloat16 *>(a.C) + at + 8 * i, make_uint4(w[0], w[1], w[2], w[3]), a.cols - col - 8 * i);
            }
        } else if (a.wide && N % 8 == 0) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                float *to = static_cast<float *>(a.C) + at + 4 * i;
                if (col + 4 * i + 4 <= a.cols) *reinterpret_cast<float4 *>(to) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                else
#pragma unroll
                    for (int t = 0; t < 4; ++t)
                        if (col + 4 * i + t < a.cols) to[t] = v[4 * i + t];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (col + i < a.cols) {
                    if (a.out_f32) static_cast<float *>(a.C)[at + i] = v[i]; else static_cast<__nv_bfloat16 *>(a.C)[at + i] = __float2bfloat16_rn(v[i]);
                }
        }
    }
}

template <int BN>
__global__ void __launch_bounds__(kThreads, BN > 128 ? 1 : 2)
linear_mx4_kernel(const __grid_constant__ CUtensorMap tm_lanes, const __grid_constant__ CUtensorMap tm_cols, Mx4Args a, int stages, uint32_t tmem_columns)
{
    using S = Shape<BN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    // codes first (1024-byte aligned), then every stage's scales
    uint8_t *scales = ring + stages * (S::kA + S::kB);
    uint64_t *bars = reinterpret_cast<uint64_t *>(ring + stages * S::kStage);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + (2 * stages + 1));
    __shared__ int s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int split = blockIdx.x % a.splits, tile = blockIdx.x / a.splits;
    const int col_tile = tile % a.col_tiles, lane_tile = tile / a.col_tiles;
    const int scale_tile = col_tile * BN / 128;             // the first one of the columns' rows
    const int n_steps = (a.blocks + kDepth / 32 - 1) / (kDepth / 32);
    const int first = (int)((long long)n_steps * split / a.splits), last = (int)((long long)n_steps * (split + 1) / a.splits);
    const uint32_t full = tc::smem_u32(bars), empty = full + 8 * stages, done = empty + 8 * stages;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { tc::mbar_init(full + 8 * s, 1); tc::mbar_init(empty + 8 * s, 1); }
        tc::mbar_init(done, 1);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 0 && lane == 0) { tc::tma_prefetch_desc(&tm_lanes); tc::tma_prefetch_desc(&tm_cols); }
    if (warp == 1) { tc::tmem_alloc(tc::smem_u32(tmem_slot), tmem_columns); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    pdl_wait();
    pdl_trigger();

    auto codes_of = [&](int s) { return tc::smem_u32(ring) + s * (S::kA + S::kB); };
    auto scales_of = [&](int s) { return tc::smem_u32(scales) + s * (S::kScaleA + S::kScaleB); };
    if (warp == 0) {
        if (lane == 0) {
            int issued = first;
            for (int k = first, s = 0, ph = 0; k < last; ++k) {
                if (!tc::mbar_wait(empty + 8 * s, (uint32_t)ph ^ 1u, &s_abort)) break;
                const uint32_t bar = full + 8 * s, part = (uint32_t)min(2, a.quads - 2 * k) * kScaleTile;   // (the last stage may hold one tile of scales)
                const bool second = S::kRowTiles == 2 && (scale_tile + 1) * 128 < a.cols;
                tc::mbar_expect_tx(bar, (uint32_t)(S::kA + S::kB) + part * (second ? 3u : 2u));
                tc::tma_load_2d(codes_of(s), &tm_lanes, k * (kCodes / 2), lane_tile * 128, bar);
                tc::tma_load_2d(codes_of(s) + S::kA, &tm_cols, k * (kCodes / 2), col_tile * BN, bar);
                bulk_load(scales_of(s), a.lane_scales + ((size_t)lane_tile * a.quads + 2 * k) * kScaleTile, part, bar);
                bulk_load(scales_of(s) + S::kScaleA, a.col_scales + ((size_t)scale_tile * a.quads + 2 * k) * kScaleTile, part, bar);
                if (second) bulk_load(scales_of(s) + 2 * S::kScaleA, a.col_scales + ((size_t)(scale_tile + 1) * a.quads + 2 * k) * kScaleTile, part, bar);
                issued = k + 1;
                if (++s == stages) { s = 0; ph ^= 1; }
            }
            if (s_abort)                                    // copies in flight get a bounded time to land before the CTA retires
                for (int k = max(first, issued - stages); k < issued; ++k) {
                    const int s = (k - first) % stages, ph = ((k - first) / stages) & 1;
                    for (int i = 0; i < (1 << 16) && !tc::mbar_try(full + 8 * s, (uint32_t)ph); ++i) {}
                }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t tmem_scales = tmem + BN, skip = (uint32_t)(col_tile * BN % 128 / 32);          // (the columns' first row in its scale tile)
        bool ok = true;
        for (int k = first, s = 0, ph = 0; k < last; ++k) {
            ok = __all_sync(0xffffffffu, tc::mbar_wait(full + 8 * s, (uint32_t)ph, &s_abort));
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t ta = tmem_scales + (uint32_t)(s * S::kScaleCols), tb = ta + 8;
            const int tiles = min(2, a.quads - 2 * k);
            for (int q = 0; q < tiles; ++q) {
                copy_scales_elect(ta + 4 * q, scales_of(s) + q * kScaleTile);
#pragma unroll
                for (int r = 0; r < S::kRowTiles; ++r) copy_scales_elect(tb + q * 4 * S::kRowTiles + 4 * r, scales_of(s) + S::kScaleA + r * 2 * kScaleTile + q * kScaleTile);
            }
            const uint64_t da = tc::smem_desc_sw128(codes_of(s)), db = tc::smem_desc_sw128(codes_of(s) + S::kA);
            const int mmas = min(4, (a.blocks - k * 8 + 1) / 2);                // 64 columns each
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < mmas)
                    mma_mxf4_elect(tmem, da + (uint64_t)(2 * i), db + (uint64_t)(2 * i), idesc_mxf4(128, BN, i & 1), ta + 4 * (i >> 1), tb + (i >> 1) * 4 * S::kRowTiles + skip,
                                   (k != first || i != 0) ? 1u : 0u);
            tc::mma_commit_elect(empty + 8 * s);
            if (++s == stages) { s = 0; ph ^= 1; }
        }
        if (ok) tc::mma_commit_elect(done);
        __syncwarp();
    }
    // ---------------- the tile: warps 2-5, each its quarter of the lanes
    const int q = warp & 3, row = q * 32 + lane;
    const bool storing = warp >= 2;
    bool ok = storing && tc::mbar_wait(done, 0, &s_abort);
    ok = __all_sync(0xffffffffu, ok);
    if (ok) tc::tc_fence_after();
    const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16);
    constexpr int CH = BN < 32 ? BN : 32;
    if (a.splits == 1) {
        if (ok) {
#pragma unroll 1
            for (int c = 0; c < BN; c += CH) {
                uint32_t u[32];
                float v[CH];
                tc::tmem_ld32(acc + c, u);                  // (a narrow tile reads columns of scales too)
                tc::tmem_ld_wait32(u);
#pragma unroll
                for (int i = 0; i < CH; ++i) v[i] = __uint_as_float(u[i]) * a.scale;
                store_columns<CH>(a, lane_tile * 128 + row, col_tile * BN + c, v);
            }
        }
    } else if constexpr (BN <= 128) {
        // partial sums to this CTA's ring (every copy into it has landed and been read by now), then each rank adds its columns of all ranks'
        float *mine = reinterpret_cast<float *>(ring);
        if (ok) {
#pragma unroll 1
            for (int c = 0; c < BN; c += CH) {
                uint32_t u[32];
                tc::tmem_ld32(acc + c, u);
                tc::tmem_ld_wait32(u);
#pragma unroll
                for (int i = 0; i < CH; ++i) mine[(c + i) * 128 + row] = __uint_as_float(u[i]);
            }
        }
        // Tensor memory is given back before the ranks wait for one another: a CTA that kept it could hold up another launch's CTA on this SM
        // whose own rank a third SM's CTA waits for.
        tc::tc_fence_before();
        __syncthreads();
        if (warp == 1) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, tmem_columns); }
        tc::cluster_sync();
        if (storing) {
            constexpr int W = BN / 8;                       // columns of a slice
            for (int slice = split; slice < 8; slice += a.splits) {
                float v[W];
#pragma unroll
                for (int i = 0; i < W; ++i) v[i] = 0.f;
                for (int r = 0; r < a.splits; ++r) {
                    const uint32_t from = tc::mapa(tc::smem_u32(mine + (slice * W) * 128 + row), (uint32_t)r);
#pragma unroll
                    for (int i = 0; i < W; ++i) v[i] += load_remote(from + i * 512);
                }
#pragma unroll
                for (int i = 0; i < W; ++i) v[i] *= a.scale;
                if (!s_abort) store_columns<W>(a, lane_tile * 128 + row, col_tile * BN + slice * W, v);
            }
        }
        tc::cluster_sync();                                 // the ring stays until every rank has read it
    }
    if (a.splits == 1) {
        tc::tc_fence_before();
        __syncthreads();
        if (warp == 1) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, tmem_columns); }
    }
    if (threadIdx.x == 0 && s_abort && a.err) atomicExch(a.err, SFS_ERR_TIMEOUT);
}

// Which operand lies on the lanes, how many rows of the other a tile has, and over how many CTAs its k-steps are divided; or persistent CTAs.
// A step costs what it takes to bring it to the SM, about 55 bytes a clock, shared by the CTAs of an SM, which is more than its MMAs take in
// every shape here; a tile 6000 clocks around its steps, a join 2500 more.
struct Tiles { bool features_on_lanes, many; int bn, splits; };
Tiles choose_tiles(int M, int N, int n_steps, bool wide)
{
    const long long sms = gemm_num_sms();
    Tiles best = {};
    double best_clk = 1e30;
    auto consider = [&](bool features_on_lanes, int bn, int splits) {
        const long long lanes = features_on_lanes ? N : M, cols = features_on_lanes ? M : N;
        const long long ctas = (lanes + 127) / 128 * ((cols + bn - 1) / bn) * splits, per_sm = bn > 128 ? 1 : 2;
        const double bytes = (std::min<double>(128, (double)lanes) + std::min<double>(bn, (double)cols)) * 136 + 1024;
        // whole rounds of the machine; the last one may leave SMs with one CTA
        const long long full = ctas / (sms * per_sm), rest = ctas - full * sms * per_sm;
        const double step = bytes / 55, steps = (double)((n_steps + splits - 1) / splits);
        const double clk = full * (steps * step * per_sm + 6000) + (rest == 0 ? 0 : steps * step * (rest > sms ? per_sm : 1) + 6000) + (splits > 1 ? 2500 : 0);
        if (clk < best_clk) { best_clk = clk; best = {features_on_lanes, false, bn, splits}; }
    };
    // Rows of C that take no wide stores: with features on the lanes a warp's stores are consecutive all the same (235 x 2177 x 112: 19.6 us
    // with tokens on the lanes, 5.7 so).
    if (M <= 128 || !wide)
        for (int splits = 1; splits <= 8 && (splits == 1 || n_steps >= 2 * splits); splits *= 2) consider(true, M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128, splits);
    if (M > 64 && wide) {
        for (int splits = 1; splits <= 8 && (splits == 1 || n_steps >= 2 * splits); splits *= 2) consider(false, 128, splits);
        consider(false, 192, 1);
        consider(false, 256, 1);
    }
    // Persistent: the next tile's stages are loaded while a tile is stored.  A step counts 700 clocks, against 968 of the same tile above, though in
    // the longest products both take about 1000: chosen by times.  Over 40 shapes of 129 to 6144 rows the choice so made is 1.4 % slower than the
    // better of both (17 % where this kernel is never taken, 15 % where it always is); the worst, short fp32 rows whose stores are not counted:
    // 1728 x 2240 x 224 10.9 us, 8.0 persistent.
    if (M > 128) {
        const long long tiles = (long long)((M + 127) / 128) * ((N + kMx4ManyCols - 1) / kMx4ManyCols), rounds = (tiles + sms - 1) / sms;
        const double clk = (double)rounds * (n_steps * 700.0 + (wide ? 2500 : 5500)) + 5000;
        if (clk < best_clk) best = {false, true, kMx4ManyCols, 1};
    }
    return best;
}

template <int BN>
int32_t launch(const Mx4Args &a, const Mx4Operands &x, cudaStream_t stream)
{
    using S = Shape<BN>;
    CUtensorMap tl, tcol;
    int32_t rc;
    // codes as 16-bit elements: 64 of them are one swizzled row of 128 bytes
    if ((rc = make_tmap_bf16(&tl, x.lanes, (uint64_t)a.lanes, (uint64_t)a.blocks * 8, (uint64_t)x.ld_lanes / 2, 128)) != SFS_OK) return rc;
    if ((rc = make_tmap_bf16(&tcol, x.cols, (uint64_t)a.cols, (uint64_t)a.blocks * 8, (uint64_t)x.ld_cols / 2, BN)) != SFS_OK) return rc;
    const long long ctas = (long long)((a.lanes + 127) / 128) * a.col_tiles * a.splits;
    SFS_REQUIRE(ctas <= 0x7FFFFFFF, SFS_ERR_UNSUPPORTED, "linear_mx4: too many tiles");
    // no more than there are steps (but room for the partial sums): what a short call leaves free lets the next launch's CTAs start beside it
    const int n_steps = (a.blocks + kDepth / 32 - 1) / (kDepth / 32);
    const int stages = std::min(S::stages(BN > 128 || ctas <= gemm_num_sms() ? 1 : 2), std::max(2, (n_steps + a.splits - 1) / a.splits));
    const size_t shared = (size_t)S::shared(stages);
    // what the instance takes at most, whatever this call takes: another thread's launch may come between this and ours
    SFS_CUDA(allow_shared(linear_mx4_kernel<BN>, (size_t)S::shared(S::stages(1))));
    if (a.splits > 1) SFS_CUDA(launch_pdl_cluster(linear_mx4_kernel<BN>, a.splits, dim3((unsigned)ctas), dim3(kThreads), shared, stream, tl, tcol, a, stages, S::tmem_columns(stages)));
    else SFS_CUDA(launch_pdl(linear_mx4_kernel<BN>, dim3((unsigned)ctas), dim3(kThreads), shared, stream, tl, tcol, a, stages, S::tmem_columns(stages)));
    return SFS_OK;
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
    int32_t *err = nullptr;
    const int32_t rc = status_word_outside_captures((cudaStream_t)stream, &err);
    if (rc != SFS_OK) return rc;

    const int n_steps = (K + kDepth - 1) / kDepth;
    const bool wide = aligned_to(d_C, 16) && ldc * (out_dtype ? 4 : 2) % 16 == 0;
    const Tiles t = choose_tiles(M, N, n_steps, wide);
    const bool features_on_lanes = t.features_on_lanes;
    const int lanes = features_on_lanes ? N : M, cols = features_on_lanes ? M : N, bn = t.bn, splits = t.splits;
    const int col_tiles = (cols + bn - 1) / bn;
    Mx4Args a = {};
    a.lane_scales = (const uint8_t *)(features_on_lanes ? d_B_scales : d_A_scales);
    a.col_scales = (const uint8_t *)(features_on_lanes ? d_A_scales : d_B_scales);
    a.C = d_C; a.ldc = ldc; a.lanes = lanes; a.cols = cols; a.blocks = (K + 31) / 32; a.quads = (K + 127) / 128;
    a.col_tiles = col_tiles; a.splits = splits; a.out_f32 = out_dtype; a.features_on_lanes = features_on_lanes; a.scale = scale; a.err = err;
    a.wide = wide; a.unit = wide ? 16 : out_dtype || (aligned_to(d_C, 4) && ldc % 2 == 0) ? 4 : 2;
    const Mx4Operands x = features_on_lanes ? Mx4Operands{d_B, d_A, ldb, lda} : Mx4Operands{d_A, d_B, lda, ldb};
    if (t.many) return linear_mx4_many(a, x, (cudaStream_t)stream);
    switch (bn) {
    case 16: return launch<16>(a, x, (cudaStream_t)stream);
    case 32: return launch<32>(a, x, (cudaStream_t)stream);
    case 64: return launch<64>(a, x, (cudaStream_t)stream);
    case 128: return launch<128>(a, x, (cudaStream_t)stream);
    case 192: return launch<192>(a, x, (cudaStream_t)stream);
    default: return launch<256>(a, x, (cudaStream_t)stream);
    }
}

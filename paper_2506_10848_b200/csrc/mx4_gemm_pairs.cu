// C = scale * A * B^T of two matrices of microscaled 4-bit numbers, many rows: a pair of CTAs (one per SM of a TPC) computes 256 x 192
// tiles with tcgen05.mma.cta_group::2 kind::mxf4, M = 256, N = 192.
//
// A single CTA's 128 x 256 tile pulls 51 KB to the SM for every 256 columns of depth, at about 55 bytes a clock twice what its MMAs take.
// In a pair each CTA brings its own 128 rows of A, half of B's rows and the scales of both, 31 KB for three quarters of the MMAs: 41 KB for
// as many.  Scales are copied to tensor memory by one instruction for both CTAs; B's scales lie in both, whole.  Persistent, with two
// accumulators, so that a tile is stored while the next one is computed (2 x 192 columns, and five stages of 24 columns of scales).
//
// Warp 0 loads, warp 1 of the leader issues, warps 2-5 store: bf16 rows pass through shared memory and leave in whole lines.
#include "mx4_gemm.cuh"
#include "tc05.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

using namespace mx4;

constexpr int kThreads = 192;
constexpr int BN = kMx4PairCols, HALF = BN / 2;
constexpr int kStages = 5;
constexpr int kA = 128 * kCodes, kB = HALF * kCodes, kScaleA = 2 * kScaleTile, kScaleB = 4 * kScaleTile;
constexpr int kStage = kA + kB + kScaleA + kScaleB;
constexpr int kScaleCols = 24;                              // of a stage: 8 of A, 16 of B
constexpr int kPark = 32 * 128;                             // a warp's 32 rows of 64 bf16 columns
constexpr int kBarriers = 2 * kStages + 4;
constexpr int kShared = kStages * kStage + 4 * 3 * kPark + 1024 + kBarriers * 8 + 16;
constexpr uint32_t kTmem = 512;
static_assert(2 * BN + kStages * kScaleCols <= (int)kTmem && (kA + kB) % 1024 == 0 && kShared <= 227 * 1024, "tile");

__device__ __forceinline__ void mma_elect(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a, uint32_t scale_b, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred P, Q;\n\telect.sync _|P, 0xffffffff;\n\tsetp.ne.b32 Q, %6, 0;\n\t"
                 "@P tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], Q;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void copy_scales_elect(uint32_t tmem, uint32_t smem)
{
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\t"
                 "@P tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(tmem), "l"(scale_desc(smem)) : "memory");
}

__global__ void __launch_bounds__(kThreads, 1)
linear_mx4_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_sa,
                       const __grid_constant__ CUtensorMap tm_sb, Mx4Args a, int row_tiles, int num_tiles)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *scales = ring + kStages * (kA + kB), *park = ring + kStages * kStage;
    uint64_t *bars = reinterpret_cast<uint64_t *>(park + 4 * 3 * kPark);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + kBarriers);
    __shared__ int s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_ctarank();            // 0: the leader, which issues
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int n_steps = (a.blocks + kDepth / 32 - 1) / (kDepth / 32);
    const uint32_t full = tc::smem_u32(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16;
    const uint32_t lead_full = tc::mapa(full, 0), lead_acc_empty = tc::mapa(acc_empty, 0);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { tc::mbar_init(full + 8 * s, 1); tc::mbar_init(empty + 8 * s, 1); }
        for (int i = 0; i < 2; ++i) { tc::mbar_init(acc_full + 8 * i, 1); tc::mbar_init(acc_empty + 8 * i, 8); }      // 2 x 4 storing warps
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 0 && lane == 0) { tc::tma_prefetch_desc(&tm_a); tc::tma_prefetch_desc(&tm_b); tc::tma_prefetch_desc(&tm_sa); tc::tma_prefetch_desc(&tm_sb); }
    if (warp == 1) { tc::tmem_alloc_2cta(tc::smem_u32(tmem_slot), kTmem); tc::tmem_relinquish_2cta(); }
    tc::tc_fence_before();
    tc::cluster_sync();                                     // barriers of both CTAs are initialised, tensor memory is allocated
    tc::tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    pdl_wait();
    pdl_trigger();

    auto codes_of = [&](uint32_t s) { return tc::smem_u32(ring) + s * (kA + kB); };
    auto scales_of = [&](uint32_t s) { return tc::smem_u32(scales) + s * (kScaleA + kScaleB); };
    if (warp == 0) {
        // ---------------- loads, each CTA its own; the bytes of both are counted on the leader's barrier
        uint32_t it = 0, s = 0, ph = 0;
        bool ok = true;
        for (int tile = pair; tile < num_tiles && ok; tile += pairs) {
            const int row_tile = tile % row_tiles * 2 + (int)rank, col0 = tile / row_tiles * BN;
            for (int k = 0; k < n_steps; ++k, ++it) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(empty + 8 * s, ph ^ 1u, &s_abort));
                if (!ok) break;
                if (rank == 0) tc::mbar_expect_tx_elect(full + 8 * s, 2u * kStage);
                const uint32_t bar = lead_full + 8 * s, to = codes_of(s), to_scales = scales_of(s);
                tc::tma_load_2d_2cta_elect(to, &tm_a, k * (kCodes / 2), row_tile * 128, bar);
                tc::tma_load_2d_2cta_elect(to + kA, &tm_b, k * (kCodes / 2), col0 + (int)rank * HALF, bar);
                // two tiles each (the second of a row's last step may be another row tile's, or zeros: no MMA reads it)
                tc::tma_load_2d_2cta_elect(to_scales, &tm_sa, 0, row_tile * a.quads + 2 * k, bar);
                tc::tma_load_2d_2cta_elect(to_scales + kScaleA, &tm_sb, 0, col0 / 128 * a.quads + 2 * k, bar);
                tc::tma_load_2d_2cta_elect(to_scales + kScaleA + 2 * kScaleTile, &tm_sb, 0, (col0 / 128 + 1) * a.quads + 2 * k, bar);
                if (++s == kStages) { s = 0; ph ^= 1u; }
            }
        }
        // every stage has been released: no signal of the tensor core is on its way to this CTA when it leaves
        if (ok)
            for (uint32_t j = it > (uint32_t)kStages ? it - kStages : 0u; j < it && tc::mbar_wait(empty + 8 * (j % kStages), (j / kStages) & 1u, &s_abort); ++j) {}
        if (s_abort && rank == 0 && lane == 0)              // copies in flight (both CTAs') get a bounded time to land before the pair retires
            for (uint32_t j = it > (uint32_t)kStages ? it - kStages : 0u; j < it; ++j)
                for (int i = 0; i < (1 << 16) && !tc::mbar_try(full + 8 * (j % kStages), (j / kStages) & 1u); ++i) {}
    } else if (warp == 1) {
        if (rank == 0) {
            uint32_t s = 0, ph = 0, lt = 0;
            bool ok = true;
            bool ready = tc::mbar_test(full, 0u);
            for (int tile = pair; tile < num_tiles && ok; tile += pairs, ++lt) {
                const uint32_t buf = lt & 1u;
                ok = __all_sync(0xffffffffu, tc::mbar_wait(acc_empty + 8 * buf, ((lt >> 1) & 1u) ^ 1u, &s_abort));     // both CTAs have stored it
                if (!ok) break;
                tc::tc_fence_after();
                const uint32_t d = tmem + buf * BN, skip = (uint32_t)(tile / row_tiles * BN % 128 / 32);
                for (int k = 0; k < n_steps; ++k) {
                    if (!ready) ready = tc::mbar_wait(full + 8 * s, ph, &s_abort);
                    ok = __all_sync(0xffffffffu, ready);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const uint32_t ns = s + 1u == (uint32_t)kStages ? 0u : s + 1u, nph = ns == 0u ? ph ^ 1u : ph;
                    ready = tc::mbar_test(full + 8 * ns, nph);
                    // scales of this stage's place in tensor memory: the MMAs that read it before have released the stage
                    const uint32_t ta = tmem + 2 * BN + s * kScaleCols, tb = ta + 8, from = scales_of(s);
                    const int tiles = min(2, a.quads - 2 * k);
                    for (int q = 0; q < tiles; ++q) {
                        copy_scales_elect(ta + 4 * q, from + q * kScaleTile);
                        copy_scales_elect(tb + 8 * q, from + kScaleA + q * kScaleTile);
                        copy_scales_elect(tb + 8 * q + 4, from + kScaleA + (2 + q) * kScaleTile);
                    }
                    const uint64_t da = tc::smem_desc_sw128(codes_of(s)), db = tc::smem_desc_sw128(codes_of(s) + kA);
                    const int mmas = min(4, (a.blocks - k * 8 + 1) / 2);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < mmas)
                            mma_elect(d, da + (uint64_t)(2 * i), db + (uint64_t)(2 * i), idesc_mxf4(256, BN, i & 1), ta + 4 * (i >> 1), tb + 8 * (i >> 1) + skip, (k | i) != 0 ? 1u : 0u);
                    tc::mma_commit_2cta_elect(empty + 8 * s);
                    s = ns; ph = nph;
                }
                tc::mma_commit_2cta_elect(acc_full + 8 * buf);                  // complete (or abandoned), both CTAs
            }
        }
    } else {
        const int q = warp & 3;
        uint32_t lt = 0;
        bool ok = true;
        uint8_t *mine = park + q * 3 * kPark;
        for (int tile = pair; tile < num_tiles && ok; tile += pairs, ++lt) {
            const uint32_t buf = lt & 1u;
            ok = __all_sync(0xffffffffu, tc::mbar_wait(acc_full + 8 * buf, (lt >> 1) & 1u, &s_abort)) && !*reinterpret_cast<volatile int *>(&s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t acc = tmem + buf * BN + ((uint32_t)(q * 32) << 16);
            const int row0 = (tile % row_tiles * 2 + (int)rank) * 128 + q * 32, col0 = tile / row_tiles * BN;
            const bool whole = !a.out_f32 && a.wide && col0 + BN <= a.cols;
#pragma unroll 1
            for (int g = 0; g < BN / 64; ++g) {             // 64 columns: 128 bytes of bf16
                uint32_t u[64];
                tc::tmem_ld32(acc + g * 64, u); tc::tmem_ld32(acc + g * 64 + 32, u + 32);
                tc::tmem_ld_wait32(u); tc::tmem_ld_wait32(u + 32);
                if (whole) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(u[8 * c + 2 * t]) * a.scale, __uint_as_float(u[8 * c + 2 * t + 1]) * a.scale);
                            w[t] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                        *reinterpret_cast<uint4 *>(mine + g * kPark + lane * 128 + ((c ^ (lane & 7)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {           // four rows at a time
                        const int r = 4 * i + (lane >> 3), c = lane & 7;
                        const uint4 v = *reinterpret_cast<const uint4 *>(mine + g * kPark + r * 128 + ((c ^ (r & 7)) * 16));
                        if (row0 + r < a.lanes) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.C) + (long long)(row0 + r) * a.ldc + col0 + g * 64 + c * 8) = v;
                    }
                } else if (row0 + lane < a.lanes) {
                    const long long at = (long long)(row0 + lane) * a.ldc + col0 + g * 64;
                    const int n = a.cols - col0 - g * 64;
                    if (a.out_f32 && a.wide && n >= 64) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            reinterpret_cast<float4 *>(static_cast<float *>(a.C) + at)[i] = make_float4(__uint_as_float(u[4 * i]) * a.scale, __uint_as_float(u[4 * i + 1]) * a.scale,
                                                                                                        __uint_as_float(u[4 * i + 2]) * a.scale, __uint_as_float(u[4 * i + 3]) * a.scale);
                    } else {
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (i < n) {
                                const float v = __uint_as_float(u[i]) * a.scale;
                                if (a.out_f32) static_cast<float *>(a.C)[at + i] = v; else static_cast<__nv_bfloat16 *>(a.C)[at + i] = __float2bfloat16_rn(v);
                            }
                    }
                }
                __syncwarp();
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0 && tile + 2 * pairs < num_tiles) tc::mbar_arrive_cluster(lead_acc_empty + 8 * buf);        // (if it is used again)
        }
    }
    // no CTA of the pair leaves while the other may still signal its barriers
    __syncwarp();
    tc::tc_fence_before();
    if (s_abort) tc::cluster_sync(); else tc::cluster_sync_relaxed();
    if (warp == 1) { tc::tc_fence_after(); tc::tmem_dealloc_2cta(tmem, kTmem); }
    if (threadIdx.x == 0 && s_abort && a.err) atomicExch(a.err, SFS_ERR_TIMEOUT);
}

}  // namespace

int32_t linear_mx4_pairs(const Mx4Args &a, const Mx4Operands &x, cudaStream_t stream)
{
    CUtensorMap ta, tb, tsa, tsb;
    int32_t rc;
    if ((rc = make_tmap_bf16(&ta, x.lanes, (uint64_t)a.lanes, (uint64_t)a.blocks * 8, (uint64_t)x.ld_lanes / 2, 128)) != SFS_OK) return rc;
    if ((rc = make_tmap_bf16(&tb, x.cols, (uint64_t)a.cols, (uint64_t)a.blocks * 8, (uint64_t)x.ld_cols / 2, HALF)) != SFS_OK) return rc;
    if ((rc = make_tmap_scale_tiles(&tsa, a.lane_scales, (uint64_t)((a.lanes + 127) / 128) * a.quads)) != SFS_OK) return rc;
    if ((rc = make_tmap_scale_tiles(&tsb, a.col_scales, (uint64_t)((a.cols + 127) / 128) * a.quads)) != SFS_OK) return rc;
    const int row_tiles = (a.lanes + kMx4PairRows - 1) / kMx4PairRows;
    const long long tiles = (long long)row_tiles * ((a.cols + BN - 1) / BN);
    SFS_REQUIRE(tiles <= 0x3FFFFFFF && ((long long)((a.lanes + 127) / 128) + 2) * a.quads <= 0x7FFFFFFF && ((long long)((a.cols + 127) / 128) + 2) * a.quads <= 0x7FFFFFFF,
                SFS_ERR_UNSUPPORTED, "linear_mx4: too many tiles");
    SFS_CUDA(allow_shared(linear_mx4_pair_kernel, kShared));
    const long long pairs = std::min<long long>(tiles, gemm_num_sms() / 2);
    SFS_CUDA(launch_pdl_cluster(linear_mx4_pair_kernel, 2, dim3((unsigned)(2 * pairs)), dim3(kThreads), (size_t)kShared, stream, ta, tb, tsa, tsb, a, row_tiles, (int)tiles));
    return SFS_OK;
}

}  // namespace sfs

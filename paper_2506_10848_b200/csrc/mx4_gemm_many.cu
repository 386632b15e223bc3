// C = scale * A * B^T of two matrices of microscaled 4-bit numbers, many tiles: one persistent CTA per SM on tiles of 128 tokens x 256
// features (tcgen05.mma kind::mxf4).
//
// Bound: a step of 256 columns of depth writes 51 KB to the SM's shared memory and its four MMAs read 48 KB of it, about 800 of a step's
// 1000 clocks at 128 bytes a clock; loads alone take 120 us of 6144 x 4096 x 12288's 142 - 155, MMAs alone 119, copying the scales 4.  What a
// CTA for every tile spends around its steps, 15000 clocks for its start, the filling of the ring and the storing of its tile, is what
// persistence saves: the next tile's stages are loaded while a tile is stored, and its MMAs begin once the accumulator has been read (us,
// 6144 x 12288 x 4096: 211 -> 164, 1536 x 12288 x 4096: 55 -> 40, 512 x 24576 x 4096: 43 -> 32).  The accumulator takes half of tensor memory and the
// stages' scales 96 columns of the rest, so there is one.  Pairs of CTAs on 256 x 256 tiles (cta_group::2) bring 35 KB a step instead, but
// copying scales for a pair kept its MMAs waiting: 171 us.
//
// Warp 0 loads, warp 1 issues, warps 2-9 store: rows pass through shared memory and leave in whole sectors, or, where they do not take
// 16-byte stores, 4 or 2 bytes of neighbouring lanes together.
#include "mx4_gemm.cuh"
#include "tc05.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

using namespace mx4;

constexpr int kStoring = 8;                                 // warps: two for each quarter of the lanes, half of the columns each
constexpr int kThreads = 64 + 32 * kStoring;
constexpr int BN = kMx4ManyCols;
constexpr int kStages = 4;
constexpr int kA = 128 * kCodes, kB = BN * kCodes, kScaleA = 2 * kScaleTile, kScaleB = 4 * kScaleTile;
constexpr int kStage = kA + kB + kScaleA + kScaleB;
constexpr int kScaleCols = 24;                              // of a stage: 8 of A, 16 of B
constexpr int kPark = 32 * 64;                              // a warp's 32 rows of 32 bf16 columns
constexpr int kBarriers = 2 * kStages + 2;
constexpr int kShared = kStages * kStage + kStoring * kPark + 1024 + kBarriers * 8 + 16;
constexpr uint32_t kTmem = 512;
static_assert(BN + kStages * kScaleCols <= (int)kTmem && (kA + kB) % 1024 == 0 && kShared <= 227 * 1024, "tile");

__global__ void __launch_bounds__(kThreads, 1)
linear_mx4_many_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, Mx4Args a, int row_tiles, int num_tiles)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *scales = ring + kStages * (kA + kB), *park = ring + kStages * kStage;
    uint64_t *bars = reinterpret_cast<uint64_t *>(park + kStoring * kPark);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + kBarriers);
    __shared__ int s_abort;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_steps = (a.blocks + kDepth / 32 - 1) / (kDepth / 32);
    const uint32_t full = tc::smem_u32(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 8;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { tc::mbar_init(full + 8 * s, 1); tc::mbar_init(empty + 8 * s, 1); }
        tc::mbar_init(acc_full, 1); tc::mbar_init(acc_empty, kStoring);
        s_abort = 0;
        tc::mbar_init_fence();
    }
    if (warp == 0 && lane == 0) { tc::tma_prefetch_desc(&tm_a); tc::tma_prefetch_desc(&tm_b); }
    if (warp == 1) { tc::tmem_alloc(tc::smem_u32(tmem_slot), kTmem); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    pdl_wait();
    pdl_trigger();

    auto codes_of = [&](uint32_t s) { return tc::smem_u32(ring) + s * (kA + kB); };
    auto scales_of = [&](uint32_t s) { return tc::smem_u32(scales) + s * (kScaleA + kScaleB); };
    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0, s = 0, ph = 0;
            bool ok = true;
            for (int tile = blockIdx.x; tile < num_tiles && ok; tile += gridDim.x) {
                const int row_tile = tile % row_tiles, col_tile = tile / row_tiles;
                const bool second = (col_tile * 2 + 1) * 128 < a.cols;
                const uint8_t *sa = a.lane_scales + (size_t)row_tile * a.quads * kScaleTile, *sb = a.col_scales + (size_t)col_tile * 2 * a.quads * kScaleTile;
                for (int k = 0; k < n_steps; ++k, ++it) {
                    ok = tc::mbar_wait(empty + 8 * s, ph ^ 1u, &s_abort);
                    if (!ok) break;
                    const uint32_t bar = full + 8 * s, part = (uint32_t)min(2, a.quads - 2 * k) * kScaleTile, to = codes_of(s), to_scales = scales_of(s);
                    tc::mbar_expect_tx(bar, (uint32_t)(kA + kB) + part * (second ? 3u : 2u));
                    tc::tma_load_2d(to, &tm_a, k * (kCodes / 2), row_tile * 128, bar);
                    tc::tma_load_2d(to + kA, &tm_b, k * (kCodes / 2), col_tile * BN, bar);
                    bulk_load(to_scales, sa + (size_t)2 * k * kScaleTile, part, bar);
                    bulk_load(to_scales + kScaleA, sb + (size_t)2 * k * kScaleTile, part, bar);
                    if (second) bulk_load(to_scales + kScaleA + 2 * kScaleTile, sb + (size_t)(a.quads + 2 * k) * kScaleTile, part, bar);
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            if (s_abort)                                    // copies in flight get a bounded time to land before the CTA retires
                for (uint32_t j = it > (uint32_t)kStages ? it - kStages : 0u; j < it; ++j)
                    for (int i = 0; i < (1 << 16) && !tc::mbar_try(full + 8 * (j % kStages), (j / kStages) & 1u); ++i) {}
        }
        __syncwarp();
    } else if (warp == 1) {
        {
            uint32_t s = 0, ph = 0, lt = 0;
            bool ok = true;
            bool ready = tc::mbar_test(full, 0u);
            for (int tile = blockIdx.x; tile < num_tiles && ok; tile += gridDim.x, ++lt) {
                ok = __all_sync(0xffffffffu, tc::mbar_wait(acc_empty, (lt & 1u) ^ 1u, &s_abort));      // the tile before has been read
                if (!ok) break;
                tc::tc_fence_after();
                for (int k = 0; k < n_steps; ++k) {
                    if (!ready) ready = tc::mbar_wait(full + 8 * s, ph, &s_abort);
                    ok = __all_sync(0xffffffffu, ready);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const uint32_t ns = s + 1u == (uint32_t)kStages ? 0u : s + 1u, nph = ns == 0u ? ph ^ 1u : ph;
                    ready = tc::mbar_test(full + 8 * ns, nph);
                    // scales of this stage's place in tensor memory: the MMAs that read it before have released the stage
                    const uint32_t ta = tmem + BN + s * kScaleCols, tb = ta + 8, from = scales_of(s);
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
                            mma_mxf4_elect(tmem, da + (uint64_t)(2 * i), db + (uint64_t)(2 * i), idesc_mxf4(128, BN, i & 1), ta + 4 * (i >> 1), tb + 8 * (i >> 1), (k | i) != 0 ? 1u : 0u);
                    tc::mma_commit_elect(empty + 8 * s);
                    s = ns; ph = nph;
                }
                tc::mma_commit_elect(acc_full);                  // complete (or abandoned)
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) / 4;
        uint32_t lt = 0;
        bool ok = true;
        uint8_t *mine = park + (warp - 2) * kPark;
        for (int tile = blockIdx.x; tile < num_tiles && ok; tile += gridDim.x, ++lt) {
            ok = __all_sync(0xffffffffu, tc::mbar_wait(acc_full, lt & 1u, &s_abort)) && !*reinterpret_cast<volatile int *>(&s_abort);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16);
            const int row0 = tile % row_tiles * 128 + q * 32, col0 = tile / row_tiles * BN;
#pragma unroll 1
            for (int g = half * (BN / 64); g < (half + 1) * (BN / 64); ++g) {          // 32 columns: 64 bytes of bf16
                uint32_t u[32];
                tc::tmem_ld32(acc + g * 32, u);
                tc::tmem_ld_wait32(u);
                if (g == (half + 1) * (BN / 64) - 1) {      // the accumulator is read: the next tile may have it while this one is stored
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(acc_empty);
                }
                // 64 bytes of a row at a time (32 columns of bf16, half of them of fp32), parked so that neighbouring lanes store neighbouring bytes
                const int passes = a.out_f32 ? 2 : 1;
#pragma unroll 1
                for (int pass = 0; pass < passes; ++pass) {
                    if (a.out_f32) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t w[4];
#pragma unroll
                            for (int t = 0; t < 4; ++t) w[t] = __float_as_uint(__uint_as_float(pass == 0 ? u[4 * c + t] : u[16 + 4 * c + t]) * a.scale);
                            *reinterpret_cast<uint4 *>(mine + lane * 64 + ((c ^ ((lane >> 1) & 3)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t w[4];
#pragma unroll
                            for (int t = 0; t < 4; ++t) {
                                const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(u[8 * c + 2 * t]) * a.scale, __uint_as_float(u[8 * c + 2 * t + 1]) * a.scale);
                                w[t] = *reinterpret_cast<const uint32_t *>(&h);
                            }
                            *reinterpret_cast<uint4 *>(mine + lane * 64 + ((c ^ ((lane >> 1) & 3)) * 16)) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                    __syncwarp();
                    const int left = (a.cols - col0 - g * 32 - pass * 16) * (a.out_f32 ? 4 : 2);               // bytes of a row from here on
                    uint8_t *to = static_cast<uint8_t *>(a.C) + ((long long)row0 * a.ldc + col0 + g * 32 + pass * 16) * (a.out_f32 ? 4 : 2);
                    const long long pitch = a.ldc * (a.out_f32 ? 4 : 2);
                    auto parked = [&](int r, int byte) { return mine + r * 64 + (((byte >> 4) ^ ((r >> 1) & 3)) * 16) + (byte & 15); };
                    const int rows = a.lanes - row0;
                    if (a.unit == 16) {                     // eight rows at a time
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = 8 * i + (lane >> 2), byte = (lane & 3) * 16;
                            if (r < rows && byte + 16 <= left) *reinterpret_cast<uint4 *>(to + r * pitch + byte) = *reinterpret_cast<const uint4 *>(parked(r, byte));
                            else if (r < rows)
                                for (int e = byte; e < min(byte + 16, left); e += 2) *reinterpret_cast<uint16_t *>(to + r * pitch + e) = *reinterpret_cast<const uint16_t *>(parked(r, e));
                        }
                    } else if (a.unit == 4) {               // two
#pragma unroll 4
                        for (int i = 0; i < 16; ++i) {
                            const int r = 2 * i + (lane >> 4), byte = (lane & 15) * 4;
                            if (r < rows && byte + 4 <= left) *reinterpret_cast<uint32_t *>(to + r * pitch + byte) = *reinterpret_cast<const uint32_t *>(parked(r, byte));
                            else if (r < rows && byte + 2 <= left) *reinterpret_cast<uint16_t *>(to + r * pitch + byte) = *reinterpret_cast<const uint16_t *>(parked(r, byte));
                        }
                    } else {
#pragma unroll 4
                        for (int r = 0; r < 32; ++r)
                            if (r < rows && lane * 2 < left) *reinterpret_cast<uint16_t *>(to + r * pitch + lane * 2) = *reinterpret_cast<const uint16_t *>(parked(r, lane * 2));
                    }
                    __syncwarp();
                }
            }
        }
    }
    __syncwarp();
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 1) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, kTmem); }
    if (threadIdx.x == 0 && s_abort && a.err) atomicExch(a.err, SFS_ERR_TIMEOUT);
}

}  // namespace

int32_t linear_mx4_many(const Mx4Args &a, const Mx4Operands &x, cudaStream_t stream)
{
    CUtensorMap ta, tb;
    int32_t rc;
    if ((rc = make_tmap_bf16(&ta, x.lanes, (uint64_t)a.lanes, (uint64_t)a.blocks * 8, (uint64_t)x.ld_lanes / 2, 128)) != SFS_OK) return rc;
    if ((rc = make_tmap_bf16(&tb, x.cols, (uint64_t)a.cols, (uint64_t)a.blocks * 8, (uint64_t)x.ld_cols / 2, BN)) != SFS_OK) return rc;
    const int row_tiles = (a.lanes + 127) / 128;
    const long long tiles = (long long)row_tiles * ((a.cols + BN - 1) / BN);
    SFS_REQUIRE(tiles <= 0x3FFFFFFF, SFS_ERR_UNSUPPORTED, "linear_mx4: too many tiles");
    SFS_CUDA(allow_shared(linear_mx4_many_kernel, kShared));
    SFS_CUDA(launch_pdl(linear_mx4_many_kernel, dim3((unsigned)std::min<long long>(tiles, gemm_num_sms())), dim3(kThreads), (size_t)kShared, stream, ta, tb, a, row_tiles, (int)tiles));
    return SFS_OK;
}

}  // namespace sfs

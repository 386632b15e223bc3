// Attention over a key / value cache of microscaled 4-bit numbers, few query rows per key head: every code is read once and decoded in
// registers, straight into the operands of mma.sync.
//
// Codes become bf16 by moving bits: the sign to the top, the three others to the low end of the exponent and the high end of the
// mantissa, which is the value times 2^-126 (0.5 as a subnormal number).  One product with 2^(c - 65) gives the value times 2^-64,
// exactly, for every scale a cache holds (65 .. 192); scores get the 2^64 back in 32 bits, values from the probabilities, which are
// taken 2^64 times as large.
//
// Tokens are the rows of the first product's tile, queries its columns: S^T = K Q^T (16 tokens x 8 queries), then O^T += V^T P^T
// (features x queries), so that a single query wastes half as much of the tensor core as it would as one row of 16.  The order of the
// features within a product is free as long as both operands agree, so a lane takes whole words of codes: of a key 32 neighbouring
// features (one scale), of values 16 neighbouring features of four tokens, whose codes are paired token by token.
//
// The tokens that any row of the CTA sees are divided over a cluster of up to 16 CTAs of 8 warps; partial outputs are joined through
// shared memory, first the warps', then the CTAs', in a fixed order: no workspace.
#include "attention_cache4.cuh"
#include "tc05.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

using mx4::cache_factor;
using mx4::codes_as_bf16;
using mx4::mul_bf16x2;

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxSplits = 16;                            // CTAs of a cluster
constexpr int kStep = 16;                                   // tokens of a warp's step
constexpr float kLazy = 8.0f;                               // the reference maximum may lag by 2^8
constexpr float kUnscale = 18446744073709551616.0f;         // 2^64

__device__ __forceinline__ void mma_bf16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ void store_remote2(uint32_t cluster_addr, float x, float y)
{
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(cluster_addr), "f"(x), "f"(y) : "memory");
}

// A warp's ring in shared memory: codes of 16 tokens a stage, copied asynchronously kDepth - 1 steps ahead.
constexpr int kDepth = 4;
template <int DH> struct Ring { static constexpr int kPart = kStep * DH / 2, kStage = 2 * kPart, kWarp = kDepth * kStage; };
__device__ __forceinline__ void copy16(uint32_t smem, const void *global) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(global) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// Row i of a tile holds token token_of(i): the four tokens whose values a quarter of the lanes read together then lie in different banks
// (with the chunks of a token's values rotated, see fetch).
__device__ __forceinline__ int token_of(int i) { return (i & 8) | ((i & 3) << 1) | ((i >> 2) & 1); }
__device__ __forceinline__ int row_of(int j) { return (j & 8) | ((j >> 1) & 3) | ((j & 1) << 2); }

// shared memory: the rings, in whose place the warps' partial outputs are joined
template <int DH, int NT> struct Few {
    static constexpr int kPartials = kWarps * 8 * NT * (DH + 4) * 4;
    static constexpr int kWork = kPartials > kWarps * Ring<DH>::kWarp ? kPartials : kWarps * Ring<DH>::kWarp;
};

template <int DH, int NT>                                   // NT tiles of 8 query rows
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1)
attention_cache4_few(Cache4Args a, int splits, int row_tiles)
{
    constexpr int ROWS = 8 * NT, KS = DH / 16, WORDS = DH / 8, BLOCKS = DH / 32;
    constexpr int MT = DH / 16;                             // feature tiles of O^T
    constexpr int PITCH = DH + 4;
    extern __shared__ __align__(16) float s_mem[];
    float *s_part = s_mem;                                  // [kWarps][ROWS][PITCH]
    float2 *s_in = reinterpret_cast<float2 *>(s_mem + Few<DH, NT>::kWork / 4);      // [splits][per], what the ranks send
    __shared__ float s_m[kWarps][ROWS], s_l[kWarps][ROWS];  // reference maximum and denominator
    __shared__ float s_cm[ROWS], s_cl[ROWS];                // of this CTA
    __shared__ float2 s_ml[kMaxSplits][ROWS];               // of all ranks: maximum (then factor) and denominator
    __shared__ float s_inv[ROWS];
    __shared__ int s_lo[ROWS], s_hi[ROWS], s_first[ROWS], s_live[ROWS];

    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rank = blockIdx.x % splits;
    int item = blockIdx.x / splits;
    const int row_tile = item % row_tiles; item /= row_tiles;
    const int kv = item % a.n_kv, b = item / a.n_kv;
    const int rows = min(ROWS, a.n_q * a.group - row_tile * ROWS);          // rows of this tile, query by query, the group's heads together
    if (splits > 1) tc::cluster_arrive_relaxed();           // (waited for before anything is sent)
    const int length = cache4_length(a, b);
    // the queries, as the second operand of S^T: lane (g, t) holds row g, the features of its words in pairs (j, j + 4)
    uint32_t q[NT][KS][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = n * 8 + g;
        const int i = (row_tile * ROWS + r) / a.group, head = kv * a.group + (row_tile * ROWS + r) % a.group;
        const __nv_bfloat16 *src = a.q + ((long long)b * a.n_q + i) * a.ld_q + (long long)head * DH + t * (DH / 4);
#pragma unroll
        for (int w = 0; w < WORDS / 4; ++w) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (r < rows) x = *reinterpret_cast<const uint4 *>(src + w * 8);
            q[n][2 * w][0] = __byte_perm(x.x, x.z, 0x5410); q[n][2 * w][1] = __byte_perm(x.x, x.z, 0x7632);
            q[n][2 * w + 1][0] = __byte_perm(x.y, x.w, 0x5410); q[n][2 * w + 1][1] = __byte_perm(x.y, x.w, 0x7632);
        }
    }
    if (threadIdx.x < ROWS) {
        Seen s = {0, 0, 0};
        int live = 0;
        if ((int)threadIdx.x < rows) {
            const int i = (row_tile * ROWS + threadIdx.x) / a.group;
            long long p = (long long)length - a.n_q + i;
            live = 1;
            if (a.positions) { p = a.positions[(long long)b * a.n_q + i]; live = p >= 0; }
            if (live) s = cache4_seen(a, length, p);
        }
        s_first[threadIdx.x] = s.first; s_lo[threadIdx.x] = s.lo; s_hi[threadIdx.x] = s.hi; s_live[threadIdx.x] = live;
    }
    __syncthreads();
    // what any row sees: [0, first) and [lo, hi); what all rows see: [all_lo, all_hi)
    int first = 0, lo = 0x7FFFFFFF, hi = 0, all_lo = 0, all_hi = 0x7FFFFFFF;
    for (int r = 0; r < rows; ++r) {
        all_lo = max(all_lo, s_lo[r]); all_hi = min(all_hi, s_hi[r]);
        if (s_hi[r] > s_lo[r] || s_first[r] > 0) { first = max(first, s_first[r]); lo = min(lo, s_lo[r]); hi = max(hi, s_hi[r]); }
    }
    lo = min(lo, hi);
    first = min(first, lo);                                 // (one row's first tokens may lie in another row's window)
    const int n_first = (first + kStep - 1) / kStep, n_steps = n_first + (hi - lo + kStep - 1) / kStep;
    const int my_first = (int)((long long)n_steps * rank / splits), my_last = (int)((long long)n_steps * (rank + 1) / splits);
    auto tokens_of = [&](int s, int &j0, int &end) {
        if (s < n_first) { j0 = s * kStep; end = first; } else { j0 = lo + (s - n_first) * kStep; end = hi; }
    };

    int r_lo[NT][2], r_hi[NT][2], r_first[NT][2];           // of rows 2 t and 2 t + 1
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) { const int r = n * 8 + 2 * t + e; r_lo[n][e] = s_lo[r]; r_hi[n][e] = s_hi[r]; r_first[n][e] = s_first[r]; }

    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) { m[n][e] = -INFINITY; l[n][e] = 0.f; }
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
    }
    const float c = a.scale_log2 * kUnscale;

    // ---- a step's codes: lane -> token lane / chunks (and + 8 with 128 features), 16-byte chunk; its scales: lane -> token lane % 16, keys' or values'
    constexpr int CHUNKS = DH / 32;                         // of a token
    const uint32_t ring = tc::smem_u32(s_mem) + warp * Ring<DH>::kWarp;
    const size_t base = (size_t)b * a.capacity * a.n_kv + kv;
    uint32_t next_scales = 0;
    auto fetch_codes = [&](int s, int stage) {
        if (s < my_last) {
            int j0, end;
            tokens_of(s, j0, end);
#pragma unroll
            for (int e = 0; e < DH / 64; ++e) {
                const int j = lane / CHUNKS + e * (32 / CHUNKS), chunk = lane % CHUNKS;
                const size_t at = (base + (size_t)min(j0 + j, end - 1) * a.n_kv) * (DH / 2) + chunk * 16;
                const uint32_t to = ring + stage * Ring<DH>::kStage;
                copy16(to + row_of(j) * (DH / 2) + chunk * 16, a.k_codes + at);
                copy16(to + Ring<DH>::kPart + j * (DH / 2) + (chunk ^ ((j >> 1) & (CHUNKS - 1))) * 16, a.v_codes + at);
            }
        }
        copies_commit();
    };
    auto fetch_scales = [&](int s) {
        if (s < my_last) {
            int j0, end;
            tokens_of(s, j0, end);
            const size_t at = base + (size_t)min(j0 + (lane & 15), end - 1) * a.n_kv;
            const uint8_t *from = (lane < 16 ? a.k_scales : a.v_scales) + at * BLOCKS;
            if constexpr (BLOCKS == 4) next_scales = *reinterpret_cast<const uint32_t *>(from);
            else next_scales = *reinterpret_cast<const uint16_t *>(from);
        }
    };

    int s = my_first + warp;
    fetch_scales(s);
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch_codes(s + d * kWarps, d);
    for (int stage = 0; s < my_last; s += kWarps, stage = stage + 1 == kDepth ? 0 : stage + 1) {
        int j0, end;
        tokens_of(s, j0, end);
        const uint32_t scales = next_scales;
        copies_wait<kDepth - 2>();
        __syncwarp();
        fetch_codes(s + (kDepth - 1) * kWarps, stage == 0 ? kDepth - 1 : stage - 1);
        fetch_scales(s + kWarps);
        const uint32_t from = ring + stage * Ring<DH>::kStage;
        uint32_t kc[2][WORDS / 4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t at = from + (g + 8 * e) * (DH / 2) + t * (DH / 8);
            if constexpr (DH == 128) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(kc[e][0]), "=r"(kc[e][1]), "=r"(kc[e][2]), "=r"(kc[e][WORDS / 4 - 1]) : "r"(at));
            else asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(kc[e][0]), "=r"(kc[e][WORDS / 4 - 1]) : "r"(at));
        }
        // ---- scores
        float sc[NT][4], sd[NT][4];                         // two chains of products
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[n][e] = sd[n][e] = 0.f;
        uint32_t f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            f[e] = cache_factor((__shfl_sync(0xffffffffu, scales, token_of(g + 8 * e)) >> (8 * (t * BLOCKS / 4))) & 255u);
            f[e] |= f[e] << 16;
        }
#pragma unroll
        for (int w = 0; w < WORDS / 4; ++w) {
            const uint32_t x0 = kc[0][w], x1 = kc[1][w];
            uint32_t A[4];
            A[0] = mul_bf16x2(codes_as_bf16<0>(x0), f[0]); A[1] = mul_bf16x2(codes_as_bf16<0>(x1), f[1]);
            A[2] = mul_bf16x2(codes_as_bf16<1>(x0), f[0]); A[3] = mul_bf16x2(codes_as_bf16<1>(x1), f[1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16(sc[n], A, q[n][2 * w][0], q[n][2 * w][1]);
            A[0] = mul_bf16x2(codes_as_bf16<2>(x0), f[0]); A[1] = mul_bf16x2(codes_as_bf16<2>(x1), f[1]);
            A[2] = mul_bf16x2(codes_as_bf16<3>(x0), f[0]); A[3] = mul_bf16x2(codes_as_bf16<3>(x1), f[1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16(sd[n], A, q[n][2 * w + 1][0], q[n][2 * w + 1][1]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[n][e] += sd[n][e];
        // ---- what the rows do not see
        const bool whole = j0 >= all_lo && j0 + kStep <= min(end, all_hi);
        if (!whole) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + token_of(g + 8 * (e >> 1));
                    const bool in = j < end && (j < r_first[n][e & 1] || (j >= r_lo[n][e & 1] && j < r_hi[n][e & 1]));
                    if (!in) sc[n][e] = -INFINITY;
                }
        }
        // ---- softmax against a reference that follows the maximum lazily
        float p[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const float x0 = fmaxf(sc[n][0], sc[n][2]) * c, x1 = fmaxf(sc[n][1], sc[n][3]) * c;
            if (__any_sync(0xffffffffu, x0 > m[n][0] + kLazy || x1 > m[n][1] + kLazy)) {
                float y[2] = {x0, x1};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) y[e] = fmaxf(y[e], __shfl_xor_sync(0xffffffffu, y[e], d));
                    const float to = fmaxf(m[n][e], y[e]), alpha = to == -INFINITY ? 1.f : tc::ex2_approx(m[n][e] - to);
                    m[n][e] = to;
                    l[n][e] *= alpha;
#pragma unroll
                    for (int j = 0; j < MT; ++j) { o[n][j][e] *= alpha; o[n][j][2 + e] *= alpha; }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float ref = m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1] - 64.f;       // probabilities times 2^64
                p[n][e] = tc::ex2_approx(fmaf(sc[n][e], c, -ref));
            }
            l[n][0] += p[n][0] + p[n][2]; l[n][1] += p[n][1] + p[n][3];
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) { pb[n][0] = transpose8(pack_bf16(p[n][0], p[n][1])); pb[n][1] = transpose8(pack_bf16(p[n][2], p[n][3])); }
        // ---- values
        // rows 2 t, 2 t + 1, 2 t + 8 and 2 t + 9 of the tile
        uint32_t fv[2], bad = 0, lo4[2][2], hi4[2][2];      // [token pair][word]: the low and the high four codes of both tokens
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int j = token_of(2 * t + 8 * e), j1 = token_of(2 * t + 1 + 8 * e);
            const uint32_t c0 = (__shfl_sync(0xffffffffu, scales, 16 + j) >> (8 * (g * BLOCKS / 8))) & 255u, c1 = (__shfl_sync(0xffffffffu, scales, 16 + j1) >> (8 * (g * BLOCKS / 8))) & 255u;
            if (c0 > mx4::kCacheHi) bad |= 1u << (2 * e);
            if (c1 > mx4::kCacheHi) bad |= 2u << (2 * e);
            fv[e] = (c0 > mx4::kCacheHi ? 0u : (c0 + 62) << 7) | (c1 > mx4::kCacheHi ? 0u : (c1 + 62) << 23);
            const uint32_t at = from + Ring<DH>::kPart;
            if constexpr (DH == 128) {
                uint32_t x, y, x1, y1;
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(at + j * 64 + (((g >> 1) ^ ((j >> 1) & 3)) * 16) + (g & 1) * 8));
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x1), "=r"(y1) : "r"(at + j1 * 64 + (((g >> 1) ^ ((j1 >> 1) & 3)) * 16) + (g & 1) * 8));
                lo4[e][0] = __byte_perm(x, x1, 0x5410); hi4[e][0] = __byte_perm(x, x1, 0x7632);
                lo4[e][1] = __byte_perm(y, y1, 0x5410); hi4[e][1] = __byte_perm(y, y1, 0x7632);
            } else {                                        // one word: its low codes are the tile's first eight features, its high codes the others
                uint32_t x, x1;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at + j * 32 + (((g >> 2) ^ ((j >> 1) & 1)) * 16) + (g & 3) * 4));
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x1) : "r"(at + j1 * 32 + (((g >> 2) ^ ((j1 >> 1) & 1)) * 16) + (g & 3) * 4));
                lo4[e][0] = __byte_perm(x, x1, 0x5410); lo4[e][1] = __byte_perm(x, x1, 0x7632);
            }
        }
        auto product = [&](auto J, int j, const uint32_t (&x)[2][2]) {
            uint32_t A[4];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int w = 0; w < 2; ++w) A[2 * e + w] = mul_bf16x2(codes_as_bf16<decltype(J)::value>(x[e][w]), fv[e]);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_bf16(o[n][j], A, pb[n][0], pb[n][1]);
        };
        product(std::integral_constant<int, 0>(), 0, lo4); product(std::integral_constant<int, 1>(), 1, lo4);
        product(std::integral_constant<int, 2>(), 2, lo4); product(std::integral_constant<int, 3>(), 3, lo4);
        if constexpr (DH == 128) {
            product(std::integral_constant<int, 0>(), 4, hi4); product(std::integral_constant<int, 1>(), 5, hi4);
            product(std::integral_constant<int, 2>(), 6, hi4); product(std::integral_constant<int, 3>(), 7, hi4);
        }
        // ---- NaN blocks reach the rows that see them, and no others: how many of them a row sees, by one more product
        if (__any_sync(0xffffffffu, bad != 0)) {
            uint32_t A[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) A[2 * e] = A[2 * e + 1] = ((bad >> (2 * e)) & 1u ? 0x3F80u : 0u) | ((bad >> (2 * e)) & 2u ? 0x3F800000u : 0u);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float in[4], count[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = j0 + token_of(g + 8 * (e >> 1));
                    in[e] = j < end && (j < r_first[n][e & 1] || (j >= r_lo[n][e & 1] && j < r_hi[n][e & 1])) ? 1.f : 0.f;
                }
                mma_bf16(count, A, transpose8(pack_bf16(in[0], in[1])), transpose8(pack_bf16(in[2], in[3])));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (count[e] != 0.f)
#pragma unroll
                        for (int j = 0; j < MT; ++j) o[n][j][e] = __uint_as_float(0x7FC00000u);
            }
        }
    }

    // ---- join the warps (their rings make room)
    copies_wait<0>();
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x = l[n][e];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            if (g == 0) { s_m[warp][n * 8 + 2 * t + e] = m[n][e]; s_l[warp][n * 8 + 2 * t + e] = x; }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {                       // rows 2 t + (e & 1); features of the lane's first or second word (or half word)
            const int r = n * 8 + 2 * t + (e & 1);
            if (r < rows)
#pragma unroll
                for (int j = 0; j < MT; ++j) s_part[(warp * ROWS + r) * PITCH + g * (DH / 8) + (e >> 1) * (DH / 16) + j] = o[n][j][e];
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < rows) {
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w][threadIdx.x]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float mw = s_m[w][threadIdx.x], fw = mw == -INFINITY ? 0.f : tc::ex2_approx(mw - M);
            L += fw * s_l[w][threadIdx.x];
            s_m[w][threadIdx.x] = fw;
        }
        s_cm[threadIdx.x] = M; s_cl[threadIdx.x] = L;
        if (splits == 1) s_inv[threadIdx.x] = L == 0.f ? 0.f : kUnscale / L;
    }
    __syncthreads();
    // ---- join the CTAs: rank k finishes the pairs of features [k per, (k + 1) per) of the tile's rows; the others send it theirs
    const int pairs = rows * DH / 2, per = (pairs + splits - 1) / splits;
    auto finish = [&](int i, float x, float y) {
        const int r = 2 * i / DH, d = 2 * i % DH;
        if (!s_live[r]) return;
        const int qi = (row_tile * ROWS + r) / a.group, head = kv * a.group + (row_tile * ROWS + r) % a.group;
        *reinterpret_cast<uint32_t *>(a.out + ((long long)b * a.n_q + qi) * a.ld_out + (long long)head * DH + d) = pack_bf16(x * s_inv[r], y * s_inv[r]);
    };
    if (splits > 1) {
        tc::cluster_wait();                                 // every rank has started: its shared memory is there
        for (int i = threadIdx.x; i < rows * splits; i += kThreads) {
            const int r = i % rows;
            store_remote2(tc::mapa(tc::smem_u32(&s_ml[rank][r]), (uint32_t)(i / rows)), s_cm[r], s_cl[r]);
        }
    }
    for (int i = threadIdx.x; i < pairs; i += kThreads) {
        const int r = 2 * i / DH, d = 2 * i % DH;
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 v = *reinterpret_cast<const float2 *>(&s_part[(w * ROWS + r) * PITCH + d]);
            x += s_m[w][r] * v.x; y += s_m[w][r] * v.y;
        }
        if (splits > 1) store_remote2(tc::mapa(tc::smem_u32(&s_in[rank * per + i % per]), (uint32_t)(i / per)), x, y);
        else finish(i, x, y);
    }
    if (splits > 1) {
        tc::cluster_sync();
        if ((int)threadIdx.x < rows) {
            float M = -INFINITY, L = 0.f;
            for (int k = 0; k < splits; ++k) M = fmaxf(M, s_ml[k][threadIdx.x].x);
            for (int k = 0; k < splits; ++k) {
                const float mk = s_ml[k][threadIdx.x].x, fk = mk == -INFINITY ? 0.f : tc::ex2_approx(mk - M);
                L += fk * s_ml[k][threadIdx.x].y;
                s_ml[k][threadIdx.x].x = fk;
            }
            s_inv[threadIdx.x] = L == 0.f ? 0.f : kUnscale / L;
        }
        __syncthreads();
        for (int p = threadIdx.x; p < per && rank * per + p < pairs; p += kThreads) {
            const int i = rank * per + p, r = 2 * i / DH;
            float x = 0.f, y = 0.f;
            for (int k = 0; k < splits; ++k) { const float2 v = s_in[k * per + p]; x += s_ml[k][r].x * v.x; y += s_ml[k][r].x * v.y; }
            finish(i, x, y);
        }
    }
}

template <int DH, int NT>
int32_t launch_few(const Cache4Args &a, cudaStream_t stream)
{
    constexpr int ROWS = 8 * NT;
    constexpr size_t shared = Few<DH, NT>::kWork + (size_t)(ROWS * DH + 2 * kMaxSplits) * 4;
    const int row_tiles = (int)(((long long)a.n_q * a.group + ROWS - 1) / ROWS);
    const long long items = (long long)a.batch * a.n_kv * row_tiles;
    // as many CTAs as the machine holds at a time, but no fewer than two steps of 16 tokens for every warp
    const int slots = gemm_num_sms() * (NT == 1 ? 2 : 1);
    int splits = 1;
    while (splits < kMaxSplits && items * splits * 2 <= slots && a.capacity > splits * kWarps * kStep * 2) splits *= 2;
    SFS_REQUIRE(items * splits <= 0x7FFFFFFF, SFS_ERR_UNSUPPORTED, "attention_cache4: too many rows and heads for one call");
    SFS_CUDA(allow_shared(attention_cache4_few<DH, NT>, shared));
    if (splits > 8) SFS_CUDA(cudaFuncSetAttribute(attention_cache4_few<DH, NT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    if (splits > 1) SFS_CUDA(launch_pdl_cluster(attention_cache4_few<DH, NT>, splits, dim3((unsigned)(items * splits)), dim3(kThreads), shared, stream, a, splits, row_tiles));
    else SFS_CUDA(launch_pdl(attention_cache4_few<DH, NT>, dim3((unsigned)items), dim3(kThreads), shared, stream, a, splits, row_tiles));
    return SFS_OK;
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
    const int64_t rows = (int64_t)n_q * a.group;
    if (rows > 16) {
        a.err = device_status_word();
        SFS_REQUIRE(a.err != nullptr, SFS_ERR_OOM, "cannot allocate the device status word");
        return attention_cache4_many(a, cache->head_dim, (cudaStream_t)stream);
    }
    const bool one = rows <= 8;
    if (cache->head_dim == 128) return one ? launch_few<128, 1>(a, (cudaStream_t)stream) : launch_few<128, 2>(a, (cudaStream_t)stream);
    return one ? launch_few<64, 1>(a, (cudaStream_t)stream) : launch_few<64, 2>(a, (cudaStream_t)stream);
}

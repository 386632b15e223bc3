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
//
// Probabilities are rounded to bf16, since an MMA takes both operands in one type: each is off by at most 2^-8 of itself, sums and outputs stay in
// 32 bits.  Outputs are then off by 0.0020 to 0.0023 (of their size, against 64 bits) where probabilities in 32 bits give 0.0017, which is what
// rounding the outputs costs; keeping the lost bits would take a second product with the values.
//
// Bound: issue slots, of which 16 tokens of a key head take 430 (280 of them decode), with the logic pipe half and the multiplying pipe 40 %
// busy; 2.9 TB/s of codes and scales (4 x 32768 tokens, 8 key heads, 32 queries' heads: 48 us; 22 at the HBM rate).  For short contexts the
// launch and the chain from lengths to scores to the join: 7.7 us for 1536 tokens of 32 heads.
#include "attention_cache4.cuh"
#include "tc05.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

using mx4::codes_as_bf16;
using mx4::mul_bf16x2;

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 8;                                    // query rows of a CTA
constexpr int kPerSm = 2;                                   // CTAs
constexpr int kMaxSplits = 16;                            // CTAs of a cluster
constexpr int kStep = 32;                                   // tokens of a warp's step, two tiles of 16
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

__device__ __forceinline__ void store_remote4(uint32_t cluster_addr, float x, float y, float z, float w)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_addr), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}

// A warp's two stages in shared memory: codes and scales of a step's tokens, the next step's copied while the present one is worked on.
// Behind them the present step's scales as factors, keys' as a pair of equal bf16 numbers per block, values' as one.
template <int DH> struct Ring {
    static constexpr int kPart = kStep * DH / 2, kScales = 2 * kPart, kStage = kScales + 2 * kStep * 4, kBlocks = DH / 32;
    static constexpr int kKeyFactors = 2 * kStage, kValueFactors = kKeyFactors + kStep * kBlocks * 4, kWarp = kValueFactors + kStep * kBlocks * 2;
};
// four bytes, of which the first `bytes` are read and the others 0
__device__ __forceinline__ void copy4(uint32_t smem, const void *global, int bytes) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem), "l"(global), "r"(bytes) : "memory"); }
// Row i of a tile of 16 holds token token_of(i): the four tokens whose values a quarter of the lanes read together then lie in different banks
// (with the chunks of a token's values rotated, see fetch).
__device__ __forceinline__ int token_of(int i) { return (i & 8) | ((i & 3) << 1) | ((i >> 2) & 1); }
__device__ __forceinline__ int row_of(int j) { return (j & 8) | ((j >> 1) & 3) | ((j & 1) << 2); }

// shared memory: the rings, in whose place the warps' partial outputs are joined
template <int DH> struct Few {
    static constexpr int kPartials = kWarps * kRows * (DH + 4) * 4;
    static constexpr int kWork = kPartials > kWarps * Ring<DH>::kWarp ? kPartials : kWarps * Ring<DH>::kWarp;
};

template <int DH>
__global__ void __launch_bounds__(kThreads, kPerSm)
attention_cache4_few(Cache4Args a, int log_splits, int row_tiles)
{
    constexpr int ROWS = kRows, WORDS = DH / 8, BLOCKS = DH / 32;
    constexpr int MT = DH / 16;                             // feature tiles of O^T
    constexpr int PITCH = DH + 4;
    extern __shared__ __align__(16) float s_mem[];
    float *s_part = s_mem;                                  // [kWarps][ROWS][PITCH]
    float4 *s_in = reinterpret_cast<float4 *>(s_mem + Few<DH>::kWork / 4);      // [splits][ROWS][DH / 2 / splits], what the ranks send
    __shared__ float2 s_ml[kWarps][ROWS];                   // reference maximum and denominator
    __shared__ int s_lo[ROWS], s_hi[ROWS], s_first[ROWS], s_live[ROWS];
    __shared__ uint4 s_q[WORDS / 4][32];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int splits = 1 << log_splits, rank = blockIdx.x & (splits - 1);
    int item = blockIdx.x >> log_splits;
    const int row_tile = item % row_tiles; item /= row_tiles;
    const int kv = item % a.n_kv, b = item / a.n_kv;
    const int rows = min(ROWS, a.n_q * a.group - row_tile * ROWS);          // rows of this tile, query by query, the group's heads together
    if (splits > 1) tc::cluster_arrive_relaxed();           // (waited for before anything is sent)
    pdl_wait();
    pdl_trigger();
    // the queries, as the second operand of S^T: lane (g, t) holds row g, the features of its words in pairs (j, j + 4)
    if (warp == 0) {
        const int r = g;
        const int i = (row_tile * ROWS + r) / a.group, head = kv * a.group + (row_tile * ROWS + r) % a.group;
        const __nv_bfloat16 *src = a.q + ((long long)b * a.n_q + i) * a.ld_q + (long long)head * DH + t * (DH / 4);
        uint4 x[WORDS / 4];
#pragma unroll
        for (int w = 0; w < WORDS / 4; ++w) x[w] = r < rows ? *reinterpret_cast<const uint4 *>(src + w * 8) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < WORDS / 4; ++w)
            s_q[w][lane] = make_uint4(__byte_perm(x[w].x, x[w].z, 0x5410), __byte_perm(x[w].x, x[w].z, 0x7632), __byte_perm(x[w].y, x[w].w, 0x5410), __byte_perm(x[w].y, x[w].w, 0x7632));
    } else if (warp == 1 && lane < ROWS) {                 // meanwhile, what the rows see
        Seen s = {0, 0, 0};
        int live = 0;
        if (lane < rows) {
            const int i = (row_tile * ROWS + lane) / a.group;
            const int given = a.positions ? a.positions[(long long)b * a.n_q + i] : 0, length = cache4_length(a, b);
            live = given >= 0;
            if (live) s = cache4_seen(a, length, a.positions ? (long long)given : (long long)length - a.n_q + i);
        }
        s_first[lane] = s.first; s_lo[lane] = s.lo; s_hi[lane] = s.hi; s_live[lane] = live;
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
    const int my_first = (int)(((long long)n_steps * rank) >> log_splits), my_last = (int)(((long long)n_steps * (rank + 1)) >> log_splits);
    auto tokens_of = [&](int s, int &j0, int &end) {
        if (s < n_first) { j0 = s * kStep; end = first; } else { j0 = lo + (s - n_first) * kStep; end = hi; }
    };

    int r_lo[2], r_hi[2], r_first[2];                       // of rows 2 t and 2 t + 1
#pragma unroll
    for (int e = 0; e < 2; ++e) { const int r = 2 * t + e; r_lo[e] = s_lo[r]; r_hi[e] = s_hi[r]; r_first[e] = s_first[r]; }

    float o[MT][4], m[2], l[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) { m[e] = -INFINITY; l[e] = 0.f; }
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    const float c = a.scale_log2 * kUnscale;

    // ---- a step's codes: lane -> token lane / chunks (+ 32 / chunks a copy), 16-byte chunk; its scales: lane -> token
    constexpr int CHUNKS = DH / 32, COPIES = DH / 32, HOP = 32 / CHUNKS;
    uint8_t *ring = reinterpret_cast<uint8_t *>(s_mem) + warp * Ring<DH>::kWarp;
    const size_t base = (size_t)b * a.capacity * a.n_kv + kv;
    const int my_token = lane / CHUNKS, my_chunk = lane % CHUNKS;
    const uint32_t token_bytes = (uint32_t)a.n_kv * (DH / 2), token_scales = (uint32_t)a.n_kv * BLOCKS;
    const uint8_t *k_from = a.k_codes + base * (DH / 2) + my_chunk * 16, *v_from = a.v_codes + base * (DH / 2) + my_chunk * 16;
    const uint32_t ring_at = tc::smem_u32(ring);
    const uint32_t k_to = ring_at + row_of(my_token) * (DH / 2) + my_chunk * 16, v_to = ring_at + Ring<DH>::kPart + my_token * (DH / 2) + (my_chunk ^ ((my_token >> 1) & (CHUNKS - 1))) * 16;
    const size_t all_scales = (size_t)a.batch * a.capacity * a.n_kv * BLOCKS;
    const int last_token = a.capacity - 1;
    auto fetch = [&](int s, uint32_t stage) {               // tokens behind the sequence are read too, but none behind the cache
        if (s < my_last) {
            int j0, end;
            tokens_of(s, j0, end);
#pragma unroll
            for (int e = 0; e < COPIES; ++e) {
                const size_t at = (size_t)(uint32_t)min(j0 + my_token + e * HOP, last_token) * token_bytes;
                copy16(k_to + stage + e * HOP * (DH / 2), k_from + at);
                copy16(v_to + stage + e * HOP * (DH / 2), v_from + at);
            }
            const size_t at = base * BLOCKS + (size_t)(uint32_t)min(j0 + lane, last_token) * token_scales;
            const uint32_t to = ring_at + stage + Ring<DH>::kScales + lane * 4;
            if constexpr (BLOCKS == 4) { copy4(to, a.k_scales + at, 4); copy4(to + kStep * 4, a.v_scales + at, 4); }
            else {                                          // four bytes are two tokens' scales: ours are one half
                const size_t at4 = at & ~(size_t)3;
                const int bytes = (int)min((size_t)4, all_scales - at4);
                copy4(to, a.k_scales + at4, bytes); copy4(to + kStep * 4, a.v_scales + at4, bytes);
            }
        }
        copies_commit();
    };

    int s = my_first + warp;
    uint32_t stage = 0;
    fetch(s, 0);
    for (; s < my_last; s += kWarps, stage = Ring<DH>::kStage - stage) {
        int j0, end;
        tokens_of(s, j0, end);
        const uint8_t *from = ring + stage;
        copies_wait();
        // Scales of this lane's token as factors 2^(c - 65), two of 16 bits from one multiplication.  Where a byte is above 192, a key's
        // factor is NaN, a value's 0, so that it does not reach the rows that do not see its token (see below).
        uint32_t scales[2], above[2], f01[2], f23[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            scales[e] = *reinterpret_cast<const volatile uint32_t *>(from + Ring<DH>::kScales + e * kStep * 4 + lane * 4);     // this lane's own copy
            if constexpr (BLOCKS == 2) {
                if (((uint32_t)base + (uint32_t)min(j0 + lane, last_token) * (uint32_t)a.n_kv) & 1) scales[e] >>= 16;
                scales[e] &= 0xFFFFu;
            }
            above[e] = ((scales[e] & 0x7F7F7F7Fu) + 0x3F3F3F3Fu) & scales[e] & 0x80808080u;
            f01[e] = (__byte_perm(scales[e], 0, 0x4140) + 0x003E003Eu) * 128u;
            f23[e] = (__byte_perm(scales[e], 0, 0x4342) + 0x003E003Eu) * 128u;
        }
        const bool any_above = __any_sync(0xffffffffu, (above[0] | above[1]) != 0);     // (and every lane has left the step before)
        if (any_above)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t instead = e == 0 ? 0x7FC0u : 0u;
                if (above[e] & 0x80u) f01[e] = (f01[e] & 0xFFFF0000u) | instead;
                if (above[e] & 0x8000u) f01[e] = (f01[e] & 0xFFFFu) | instead << 16;
                if (above[e] & 0x800000u) f23[e] = (f23[e] & 0xFFFF0000u) | instead;
                if (above[e] & 0x80000000u) f23[e] = (f23[e] & 0xFFFFu) | instead << 16;
            }
        __syncwarp();
        {
            uint8_t *kf = ring + Ring<DH>::kKeyFactors + ((lane & 16) | row_of(lane & 15)) * BLOCKS * 4, *vf = ring + Ring<DH>::kValueFactors + lane * BLOCKS * 2;
            const uint32_t a0 = __byte_perm(f01[0], 0, 0x1010), a1 = __byte_perm(f01[0], 0, 0x3232);
            if constexpr (BLOCKS == 4) {
                *reinterpret_cast<uint4 *>(kf) = make_uint4(a0, a1, __byte_perm(f23[0], 0, 0x1010), __byte_perm(f23[0], 0, 0x3232));
                *reinterpret_cast<uint2 *>(vf) = make_uint2(f01[1], f23[1]);
            } else {
                *reinterpret_cast<uint2 *>(kf) = make_uint2(a0, a1);
                *reinterpret_cast<uint32_t *>(vf) = f01[1];
            }
        }
        __syncwarp();                                       // codes and factors of all lanes are there
        fetch(s + kWarps, Ring<DH>::kStage - stage);
        // ---- scores of both tiles
        uint32_t kc[2][2][WORDS / 4], f[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 16 * h + g + 8 * e;
                const uint8_t *at = from + r * (DH / 2) + t * (DH / 8);
                if constexpr (DH == 128) { const uint4 x = *reinterpret_cast<const uint4 *>(at); kc[h][e][0] = x.x; kc[h][e][1] = x.y; kc[h][e][WORDS / 4 - 2] = x.z; kc[h][e][WORDS / 4 - 1] = x.w; }
                else { const uint2 x = *reinterpret_cast<const uint2 *>(at); kc[h][e][0] = x.x; kc[h][e][1] = x.y; }
                f[h][e] = *reinterpret_cast<const uint32_t *>(ring + Ring<DH>::kKeyFactors + (r * BLOCKS + t * BLOCKS / 4) * 4);
            }
        float sc[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[h][e] = 0.f;
#pragma unroll
        for (int w = 0; w < WORDS / 4; ++w) {
            const uint4 q = s_q[w][lane];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t x0 = kc[h][0][w], x1 = kc[h][1][w];
                uint32_t A[4];
                A[0] = mul_bf16x2(codes_as_bf16<0>(x0), f[h][0]); A[1] = mul_bf16x2(codes_as_bf16<0>(x1), f[h][1]);
                A[2] = mul_bf16x2(codes_as_bf16<1>(x0), f[h][0]); A[3] = mul_bf16x2(codes_as_bf16<1>(x1), f[h][1]);
                mma_bf16(sc[h], A, q.x, q.y);
                A[0] = mul_bf16x2(codes_as_bf16<2>(x0), f[h][0]); A[1] = mul_bf16x2(codes_as_bf16<2>(x1), f[h][1]);
                A[2] = mul_bf16x2(codes_as_bf16<3>(x0), f[h][0]); A[3] = mul_bf16x2(codes_as_bf16<3>(x1), f[h][1]);
                mma_bf16(sc[h], A, q.z, q.w);
            }
        }
        // ---- what the rows do not see
        auto sees = [&](int h, int e) {
            const int j = j0 + 16 * h + token_of(g + 8 * (e >> 1));
            return j < end && (j < r_first[e & 1] || (j >= r_lo[e & 1] && j < r_hi[e & 1]));
        };
        if (!(j0 >= all_lo && j0 + kStep <= min(end, all_hi))) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!sees(h, e)) sc[h][e] = -INFINITY;
        }
        // ---- softmax against a reference that follows the maximum lazily
        uint32_t pb[2][2];
        {
            const float x0 = fmaxf(fmaxf(sc[0][0], sc[0][2]), fmaxf(sc[1][0], sc[1][2])) * c;
            const float x1 = fmaxf(fmaxf(sc[0][1], sc[0][3]), fmaxf(sc[1][1], sc[1][3])) * c;
            if (__any_sync(0xffffffffu, x0 > m[0] + kLazy || x1 > m[1] + kLazy)) {
                float y[2] = {x0, x1};
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) y[e] = fmaxf(y[e], __shfl_xor_sync(0xffffffffu, y[e], d));
                    const float to = fmaxf(m[e], y[e]), alpha = to == -INFINITY ? 1.f : tc::ex2_approx(m[e] - to);
                    m[e] = to;
                    l[e] *= alpha;
#pragma unroll
                    for (int j = 0; j < MT; ++j) { o[j][e] *= alpha; o[j][2 + e] *= alpha; }
                }
            }
            float ref[2];                                   // probabilities times 2^64
#pragma unroll
            for (int e = 0; e < 2; ++e) ref[e] = m[e] == -INFINITY ? 0.f : 64.f - m[e];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = tc::ex2_approx(fmaf(sc[h][e], c, ref[e & 1]));
                l[0] += p[0] + p[2]; l[1] += p[1] + p[3];
                pb[h][0] = transpose8(pack_bf16(p[0], p[1])); pb[h][1] = transpose8(pack_bf16(p[2], p[3]));
            }
        }
        // ---- values: rows 2 t, 2 t + 1, 2 t + 8 and 2 t + 9 of either tile
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t fv[2], lo4[2][2], hi4[2][2];           // [token pair][word]: the low and the high four codes of both tokens
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int j = 16 * h + token_of(2 * t + 8 * e), j1 = 16 * h + token_of(2 * t + 1 + 8 * e);
                const uint8_t *at_f = ring + Ring<DH>::kValueFactors + (g * BLOCKS / 8) * 2, *at = from + Ring<DH>::kPart;
                fv[e] = (uint32_t)*reinterpret_cast<const uint16_t *>(at_f + j * BLOCKS * 2) | (uint32_t)*reinterpret_cast<const uint16_t *>(at_f + j1 * BLOCKS * 2) << 16;
                if constexpr (DH == 128) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(at + j * 64 + (((g >> 1) ^ ((j >> 1) & 3)) * 16) + (g & 1) * 8);
                    const uint2 y = *reinterpret_cast<const uint2 *>(at + j1 * 64 + (((g >> 1) ^ ((j1 >> 1) & 3)) * 16) + (g & 1) * 8);
                    lo4[e][0] = __byte_perm(x.x, y.x, 0x5410); hi4[e][0] = __byte_perm(x.x, y.x, 0x7632);
                    lo4[e][1] = __byte_perm(x.y, y.y, 0x5410); hi4[e][1] = __byte_perm(x.y, y.y, 0x7632);
                } else {                                    // one word: its low codes are the tile's first eight features, its high codes the others
                    const uint32_t x = *reinterpret_cast<const uint32_t *>(at + j * 32 + (((g >> 2) ^ ((j >> 1) & 1)) * 16) + (g & 3) * 4);
                    const uint32_t y = *reinterpret_cast<const uint32_t *>(at + j1 * 32 + (((g >> 2) ^ ((j1 >> 1) & 1)) * 16) + (g & 3) * 4);
                    lo4[e][0] = __byte_perm(x, y, 0x5410); lo4[e][1] = __byte_perm(x, y, 0x7632);
                }
            }
            auto product = [&](auto J, int j, const uint32_t (&x)[2][2]) {
                uint32_t A[4];
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int w = 0; w < 2; ++w) A[2 * e + w] = mul_bf16x2(codes_as_bf16<decltype(J)::value>(x[e][w]), fv[e]);
                mma_bf16(o[j], A, pb[h][0], pb[h][1]);
            };
            product(std::integral_constant<int, 0>(), 0, lo4); product(std::integral_constant<int, 1>(), 1, lo4);
            product(std::integral_constant<int, 2>(), 2, lo4); product(std::integral_constant<int, 3>(), 3, lo4);
            if constexpr (DH == 128) {
                product(std::integral_constant<int, 0>(), 4, hi4); product(std::integral_constant<int, 1>(), 5, hi4);
                product(std::integral_constant<int, 2>(), 6, hi4); product(std::integral_constant<int, 3>(), 7, hi4);
            }
        }
        // ---- NaN blocks reach the rows that see them, and no others: how many of them a row sees, by one more product
        if (any_above) {
            const uint32_t bit = 0x80u << (8 * (g * BLOCKS / 8));
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                uint32_t A[4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t b0 = __shfl_sync(0xffffffffu, above[1], 16 * h + token_of(2 * t + 8 * e)) & bit, b1 = __shfl_sync(0xffffffffu, above[1], 16 * h + token_of(2 * t + 1 + 8 * e)) & bit;
                    A[2 * e] = A[2 * e + 1] = (b0 ? 0x3F80u : 0u) | (b1 ? 0x3F800000u : 0u);
                }
                float in[4], count[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e) in[e] = sees(h, e) ? 1.f : 0.f;
                mma_bf16(count, A, transpose8(pack_bf16(in[0], in[1])), transpose8(pack_bf16(in[2], in[3])));
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (count[e] != 0.f)
#pragma unroll
                        for (int j = 0; j < MT; ++j) o[j][e] = __uint_as_float(0x7FC00000u);
            }
        }
    }

    // ---- join the warps (their rings make room)
    copies_wait();
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        float x = l[e];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (g == 0) s_ml[warp][2 * t + e] = make_float2(m[e], x);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {                           // rows 2 t + (e & 1); features of the lane's first or second word (or half word)
        const int r = 2 * t + (e & 1);
        if (r < rows)
#pragma unroll
            for (int j = 0; j < MT; ++j) s_part[(warp * ROWS + r) * PITCH + g * (DH / 8) + (e >> 1) * (DH / 16) + j] = o[j][e];
    }
    __syncthreads();
    auto finish = [&](int r, int pair, float x, float y, float den) {
        if (!s_live[r]) return;
        const float inv = den == 0.f && s_hi[r] <= s_lo[r] && s_first[r] <= 0 ? 0.f : kUnscale / den;     // (0 / 0, a NaN, for scores of -inf alone)
        const int qi = (row_tile * ROWS + r) / a.group, head = kv * a.group + (row_tile * ROWS + r) % a.group;
        *reinterpret_cast<uint32_t *>(a.out + ((long long)b * a.n_q + qi) * a.ld_out + (long long)head * DH + 2 * pair) = pack_bf16(x * inv, y * inv);
    };
    constexpr int PAIRS = DH / 2;                           // of a row
    if (splits > 1) tc::cluster_wait();                     // every rank has started: its shared memory is there
    // rank k finishes the pairs [k PAIRS / splits, (k + 1) PAIRS / splits) of every row: the others send it theirs, with maximum and denominator
    for (int i = threadIdx.x; i < rows * PAIRS; i += kThreads) {
        const int r = i / PAIRS, pair = i % PAIRS;
        float mw[kWarps], M = -INFINITY, L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { mw[w] = s_ml[w][r].x; M = fmaxf(M, mw[w]); }
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float f = mw[w] == -INFINITY ? 0.f : tc::ex2_approx(mw[w] - M);
            const float2 v = *reinterpret_cast<const float2 *>(&s_part[(w * ROWS + r) * PITCH + 2 * pair]);
            L += f * s_ml[w][r].y; x += f * v.x; y += f * v.y;
        }
        if (splits == 1) { finish(r, pair, x, y, L); continue; }
        const int to = (pair << log_splits) / PAIRS, width = PAIRS >> log_splits;
        store_remote4(tc::mapa(tc::smem_u32(&s_in[(rank * ROWS + r) * width + (pair & (width - 1))]), (uint32_t)to), x, y, M, L);
    }
    if (splits > 1) {
        tc::cluster_sync();
        const int width = PAIRS >> log_splits;
        for (int i = threadIdx.x; i < rows * width; i += kThreads) {
            const int r = i / width, p = i & (width - 1);
            float M = -INFINITY, L = 0.f, x = 0.f, y = 0.f;
#pragma unroll 8
            for (int k = 0; k < splits; ++k) M = fmaxf(M, s_in[(k * ROWS + r) * width + p].z);
#pragma unroll 8
            for (int k = 0; k < splits; ++k) {
                const float4 v = s_in[(k * ROWS + r) * width + p];
                const float f = v.z == -INFINITY ? 0.f : tc::ex2_approx(v.z - M);
                L += f * v.w; x += f * v.x; y += f * v.y;
            }
            finish(r, rank * width + p, x, y, L);
        }
    }
}

// How the tokens are divided: one wave of CTAs, whole steps for every warp.  (Clusters do not cross the GPU's partitions: an eighth of the
// SMs' places stays out of their reach.)
int splits_of(long long items, long long tokens)
{
    int log_splits = 0;
    while ((1 << log_splits) < kMaxSplits && (items << (log_splits + 1)) <= (long long)gemm_num_sms() * kPerSm * 7 / 8 && tokens >= (kWarps * kStep) << (log_splits + 1)) ++log_splits;
    return log_splits;
}

// Microseconds of a call here, to choose between this kernel and the tensor-memory one: 4.5 for start and join, 2 (one CTA on an SM) or
// 2.75 (two) for a step of 32 tokens of a warp.  attention_cache4_many_us is the other side, with what both measured.
double few_us(long long items, long long tokens, int log_splits)
{
    const long long ctas = items << log_splits, sms = gemm_num_sms(), rounds = (ctas + sms * kPerSm - 1) / (sms * kPerSm);
    const long long steps = (tokens + ((long long)(kWarps * kStep) << log_splits) - 1) / ((long long)(kWarps * kStep) << log_splits);
    return (ctas <= sms ? 2.0 : 2.75) * (double)steps * rounds + 4.5;
}

template <int DH>
int32_t launch_few(const Cache4Args &a, int row_tiles, int log_splits, cudaStream_t stream)
{
    constexpr size_t shared = Few<DH>::kWork + (size_t)kRows * (DH / 2) * 16;
    const long long ctas = ((long long)a.batch * a.n_kv * row_tiles) << log_splits;
    SFS_REQUIRE(ctas <= 0x7FFFFFFF, SFS_ERR_UNSUPPORTED, "attention_cache4: too many rows and heads for one call");
    SFS_CUDA(allow_shared(attention_cache4_few<DH>, shared));
    if (log_splits > 3) SFS_CUDA(cudaFuncSetAttribute(attention_cache4_few<DH>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    if (log_splits > 0) SFS_CUDA(launch_pdl_cluster(attention_cache4_few<DH>, 1 << log_splits, dim3((unsigned)ctas), dim3(kThreads), shared, stream, a, log_splits, row_tiles));
    else SFS_CUDA(launch_pdl(attention_cache4_few<DH>, dim3((unsigned)ctas), dim3(kThreads), shared, stream, a, log_splits, row_tiles));
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
    SFS_REQUIRE((int64_t)n_q * (n_heads / cache->n_kv_heads) <= 0x7FFFFF00, SFS_ERR_UNSUPPORTED, "attention_cache4: too many rows of one key head");
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
    const int64_t rows = (int64_t)n_q * a.group, heads = (int64_t)cache->batch * cache->n_kv_heads;
    // tokens that a row sees at most, the rows being neighbours where there is a window
    const int64_t tokens = left >= 0 && right >= 0 ? std::min<int64_t>(cache->capacity, (int64_t)left + right + n_q + sinks) : cache->capacity;
    const int64_t row_tiles = (rows + kRows - 1) / kRows;
    const int log_splits = splits_of(heads * row_tiles, tokens);
    if (rows > kRows && attention_cache4_many_us(a, tokens, cache->head_dim) < few_us(heads * row_tiles, tokens, log_splits)) {
        const int32_t rc = status_word_outside_captures((cudaStream_t)stream, &a.err);
        return rc != SFS_OK ? rc : attention_cache4_many(a, tokens, cache->head_dim, (cudaStream_t)stream);
    }
    // The few-row kernel takes no status word, but the first call of either makes it: a caller who captures a call of many rows next does
    // not know which of the two a shape gets.
    if (device_status_word_if_any() == nullptr) {
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        SFS_CUDA(cudaStreamIsCapturing((cudaStream_t)stream, &capture));
        if (capture == cudaStreamCaptureStatusNone) SFS_REQUIRE(device_status_word() != nullptr, SFS_ERR_OOM, "cannot allocate the device status word");
    }
    return cache->head_dim == 128 ? launch_few<128>(a, (int)row_tiles, log_splits, (cudaStream_t)stream) : launch_few<64>(a, (int)row_tiles, log_splits, (cudaStream_t)stream);
}

// Attention over a key / value cache of microscaled 4-bit numbers, many query rows per key head: the products run on the fifth-generation
// tensor cores (tcgen05, accumulators in tensor memory), keys and values are decoded once per CTA into the operands' shared-memory layout.
//
// A CTA has two streams of 128 rows x 128-key tiles, so that the tensor core works on one while the other is in its softmax: two row tiles
// that share every decoded key and value tile (PAIR), or the even and the odd key tiles of one row tile.  A row is a (query, head) pair of
// the key head's group.  The first 8 or 16 warps decode: blocks of keys' codes, whose words of 8 features become 16-byte chunks of the
// 128-byte-swizzled K-major tile (the order of features within a word is that of the decoding, the same for queries), then a piece of eight
// tokens' values, which comes out transposed, eight tokens of a feature to a chunk.  The codes of the next tile are in flight meanwhile.
// The next eight are the softmax of the streams, one thread per row, the last issues the MMAs.
//
// Decoded values are exact: bits moved into bf16 (times 2^-126), one product with 2^(c - 65), so a common factor of 2^-64 remains, which
// scores get back in 32 bits and values from the probabilities, taken 2^64 times as large.  Probabilities are rounded to bf16 for the same
// reason and with the same effect as in the few-row kernel: an MMA's operands have one type; outputs off by 0.0020 to 0.0023 instead of 0.0017.
//
// Bound, where row tiles share what is decoded: the softmax warps' chain (scores, maximum, exponentials, hand-over: 3300 clocks of a tile,
// which the decoding warps stretch by sharing the pipes) with the MMAs behind it (1300), about 5000 clocks for a tile of both streams.
// Alone, the decoders: 3300 clocks of a tile, 16 instructions for a word of 8 codes; issue 51 % busy, shared memory 39 %, tensor pipe 22 %.
// Measured, 32 heads of 128, us: 2048 rows over 2048 tokens 94 (attention_kernel on bf16 values 73), 72 rows over 4 x 5344 87, 128 rows
// over 1536 13.9.  Scores of the next tile's second half issued while this one's is in its softmax: 118 instead of 97, MMAs of 64 keys
// read the queries twice as often.
//
// Only key tiles that some row sees are visited.  With few CTAs the tiles are divided over a cluster of up to 8, whose partial outputs
// meet in shared memory, in rank order.
#include "attention_cache4.cuh"
#include "tc05.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

using mx4::cache_factor;
using mx4::codes_as_bf16;
using mx4::mul_bf16x2;

constexpr int kDecoders = 256;                              // threads that decode keys, and those that decode values: the same, or others
// Warps: 8 or 16 that decode, 2 x 4 for the softmax, one for the MMAs.  Pairs of row tiles of 128 features want their decoding in the
// background: warps for keys and others for values (2048 rows over 2048 tokens, 32 heads: 97 us, 105 with the same; 5440 over 4096, 12
// heads: 176 and 166).  Registers: the launch's share is what the warps of a quarter of the SM can have, seven or five; the decoders give
// some to the softmax, four or two of them to two in each quarter, so that each quarter has what it needs.
template <int DH, bool PAIR>
struct Roles {
    static constexpr bool kApart = DH == 128 && PAIR;
    static constexpr int kSoftmaxWarp = kApart ? 16 : 8, kMmaWarp = kSoftmaxWarp + 8, kThreads = (kMmaWarp + 1) * 32;
    static constexpr int kRegs = kApart ? 72 : 96, kDecodeRegs = kApart ? 40 : DH == 64 ? 56 : 64, kSoftmaxRegs = kApart || DH == 64 ? 136 : 128;
    static_assert(kSoftmaxWarp / 4 * kDecodeRegs + 2 * kSoftmaxRegs <= (kSoftmaxWarp / 4 + 2) * kRegs, "what is taken was given or is free");
};
constexpr int QT = 128;                                     // rows of a stream
constexpr int KT = 128;                                     // keys of a tile
constexpr int kStages = 2;
constexpr int kBars = 4 * kStages + 8;                      // K full / empty, V full / empty, S (two), P (two halves of two), exchange, Q
constexpr float kLazy = 8.0f;
constexpr float kUnscale = 18446744073709551616.0f;         // 2^64

__device__ __forceinline__ void store_chunk(uint32_t smem, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(smem), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// Loads that keep out of the first-level cache: next to this much shared memory it has 28 KB, in lines of 128 bytes, of which a token's
// codes and scales would each take one for as long as they are under way.
__device__ __forceinline__ uint4 load16(const uint8_t *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t load1(const uint8_t *p)
{
    uint32_t v;
    asm volatile("ld.global.L1::no_allocate.u8 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float4 load_remote4(uint32_t cluster_addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 load_remote2(uint32_t cluster_addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_addr) : "memory");
    return v;
}
// bits k of [0, 64) with from <= k < to
__device__ __forceinline__ unsigned long long bit_range(int from, int to)
{
    from = min(max(from, 0), 64); to = min(max(to, 0), 64);
    const unsigned long long below_to = to >= 64 ? ~0ull : (1ull << to) - 1, below_from = from >= 64 ? ~0ull : (1ull << from) - 1;
    return below_to & ~below_from;
}

template <int DH, bool PAIR>
__global__ void __launch_bounds__(Roles<DH, PAIR>::kThreads, 1)
attention_cache4_many_kernel(Cache4Args a, int log_splits, int row_tiles)
{
    using R = Roles<DH, PAIR>;
    constexpr int kSoftmaxWarp = R::kSoftmaxWarp, kMmaWarp = R::kMmaWarp, kThreads = R::kThreads;
    constexpr int NQ = PAIR ? 2 : 1;
    constexpr int KB = DH / 64, WORDS = DH / 8, BLOCKS = DH / 32;
    constexpr int Q_BYTES = QT * DH * 2, K_BYTES = KT * DH * 2, V_BYTES = DH * KT * 2;
    constexpr int ROWS = NQ * QT;
    constexpr int RAW = DH / 2 + 16;                        // a token's codes of values as they lie in the cache; odd in 16 bytes
    constexpr int RAW8 = 8 * RAW + DH / 2, RAW_BYTES = KT / 8 * RAW8;
    constexpr uint32_t TMEM_COLS = 512;                     // S / P and O of each stream: 2 x (128 + DH) columns

    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t *sQ = smem, *sK = smem + NQ * Q_BYTES, *sV = sK + kStages * K_BYTES, *sRaw = sV + kStages * V_BYTES;
    uint64_t *bars = reinterpret_cast<uint64_t *>(sRaw + 2 * RAW_BYTES);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + kBars);
    const uint32_t s_o = tc::smem_u32(sV);                  // [QT][DH / 4] float4, this rank's output once all its MMAs are done
    __shared__ int s_abort, s_any_bad, s_range[3];          // first, lo, hi over the CTA's rows
    __shared__ int s_lo[ROWS], s_hi[ROWS], s_first[ROWS], s_query[ROWS];          // s_query: a row's query; its head in the group is what is left
    __shared__ uint8_t s_bad[4][BLOCKS][KT / 8];            // tokens whose values are NaN, by tile (four in turn) and block of features
    __shared__ __align__(16) uint16_t s_factor[2][BLOCKS][KT];     // of values' scales, by tile (two in turn), block and token
    __shared__ float s_max[2][QT], s_den[2][QT];
    __shared__ float2 s_ml[QT];                             // with its maxima and denominators
    __shared__ uint32_t s_nan[2][QT];
    __shared__ bool s_sees[ROWS];                           // rows that see some key

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int splits = 1 << log_splits, rank = blockIdx.x & (splits - 1);
    int item = blockIdx.x >> log_splits;
    const int row0 = (item % row_tiles) * ROWS; item /= row_tiles;
    const int kv = item % a.n_kv, b = item / a.n_kv;
    const int n_rows = a.n_q * a.group - row0;              // rows from this CTA's first on

    const uint32_t bar_kfull = tc::smem_u32(bars), bar_kempty = bar_kfull + 8 * kStages;
    const uint32_t bar_vfull = bar_kempty + 8 * kStages, bar_vempty = bar_vfull + 8 * kStages;
    const uint32_t bar_s = bar_vempty + 8 * kStages /* two */, bar_p = bar_s + 16 /* + 16 w + 8 half */, bar_x = bar_s + 48, bar_q = bar_s + 56;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            tc::mbar_init(bar_kfull + 8 * s, kDecoders); tc::mbar_init(bar_kempty + 8 * s, 1);
            tc::mbar_init(bar_vfull + 8 * s, kDecoders); tc::mbar_init(bar_vempty + 8 * s, 1);
        }
        for (int w = 0; w < 2; ++w) { tc::mbar_init(bar_s + 8 * w, 1); tc::mbar_init(bar_p + 16 * w, QT); tc::mbar_init(bar_p + 16 * w + 8, QT); }
        tc::mbar_init(bar_x, 2 * QT); tc::mbar_init(bar_q, 2 * QT);
        s_abort = 0; s_any_bad = 0;
        s_range[0] = 0; s_range[1] = 0x7FFFFFFF; s_range[2] = 0;
        tc::mbar_init_fence();
    }
    if (warp == kMmaWarp) { tc::tmem_alloc(tc::smem_u32(tmem_slot), TMEM_COLS); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t *>(tmem_slot);
    const uint32_t tmem_S = tmem_base, tmem_O = tmem_base + 2 * KT;          // stream w: + w * KT, + w * DH

    pdl_wait();
    pdl_trigger();
    // The softmax warps send the queries on their way before anything else is known (256 rows in a window, 8 x 32 heads: 46.2 us without, 42.1
    // with); neighbouring lanes have a row's words.
    constexpr int ROWS_AT_ONCE = 2 * QT / WORDS, BATCH = ROWS / ROWS_AT_ONCE;
    const int q_word = threadIdx.x % WORDS, q_row = (threadIdx.x - kSoftmaxWarp * 32) / WORDS;
    auto q_place = [&](int rq) { return tc::smem_u32(sQ) + rq / QT * Q_BYTES + (q_word / 8) * (QT * 128) + rq % QT * 128 + (((q_word % 8) ^ (rq & 7)) * 16); };
    if (warp >= kSoftmaxWarp && warp < kMmaWarp) {
#pragma unroll 4
        for (int k = 0; k < BATCH; ++k) {
            const int rq = q_row + k * ROWS_AT_ONCE, r = min(row0 + rq, a.n_q * a.group - 1), i = a.group == 1 ? r : r / a.group;
            copy16(q_place(rq), a.q + ((long long)b * a.n_q + i) * a.ld_q + (long long)(kv * a.group + r - i * a.group) * DH + q_word * 8, rq < n_rows ? 16 : 0);
        }
        copies_commit();
    }
    if (warp < ROWS / 32) {
        const int r = threadIdx.x;
        Seen s = {0, 0, 0};
        bool live = r < n_rows;
        const int i = (row0 + r) / a.group;
        s_query[r] = i;
        if (live) {
            const int given = a.positions ? a.positions[(long long)b * a.n_q + i] : 0, length = cache4_length(a, b);
            live = given >= 0;
            if (live) s = cache4_seen(a, length, a.positions ? (long long)given : (long long)length - a.n_q + i);
        }
        s_lo[r] = s.lo; s_hi[r] = s.hi; s_first[r] = live ? s.first : -1;      // -1: a row that is left as it was
        const bool some = s.hi > s.lo || s.first > 0;
        s_sees[r] = some;
        const int f = warp_max_i32(s.first), l = warp_min_i32(some ? s.lo : 0x7FFFFFFF), h = warp_max_i32(s.hi);
        if (lane == 0) { atomicMax(&s_range[0], f); atomicMin(&s_range[1], l); atomicMax(&s_range[2], h); }
    }
    __syncthreads();
    // The tokens that some row sees, in one sequence without the gap behind the first ones: v stands for token v below `first`, for
    // v + gap from there on.  (A row's first tokens beyond another row's window start: then lo = first, and there is no gap.)
    const int hi = s_range[2], lo = min(s_range[1], hi), first = min(s_range[0], lo), gap = lo - first, n_seen = hi - gap;
    const int n_all = (n_seen + KT - 1) / KT;
    const int tile0 = (n_all * rank) >> log_splits, n_tiles = ((n_all * (rank + 1)) >> log_splits) - tile0;         // (at most 2^24 tiles)
    auto tile_start = [&](int j) { return (j + tile0) * KT; };
    // where a row's query and output lie, without the head dimension's offset
    auto row_of = [&](int r, long long ld) { const int i = s_query[r]; return ((long long)b * a.n_q + i) * ld + (long long)(kv * a.group + row0 + r - i * a.group) * DH; };
    // what a row's sum is multiplied by: zeros only where it sees no key (scores of -inf alone are 0 times infinity, a NaN)
    auto inverse = [&](int r, float den) { return den == 0.f && !s_sees[r] ? 0.f : kUnscale / den; };
    auto token = [&](int v) { v = min(v, n_seen - 1); return v < first ? v : v + gap; };
    const int share = QT >> log_splits;                          // rows of a rank's part of the join
    const int n_streams = PAIR ? (n_tiles == 0 ? 0 : n_rows > QT ? 2 : 1) : min(n_tiles, 2);
    auto tiles_of = [&](int w) { return w >= n_streams ? 0 : (PAIR ? n_tiles : (n_tiles - w + 1) / 2); };
    auto key_tile = [&](int w, int i) { return PAIR ? i : 2 * i + w; };

    const size_t base = (size_t)b * a.capacity * a.n_kv + kv;
    if (warp < kSoftmaxWarp) {
        // ---------------- decoding, the codes of the next tile in flight.  Keys: a thread has a block of one or two keys.  Values: a piece of
        // eight tokens (8 ct .. of half kb of the tile) by a word of features, which comes out transposed.
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R::kDecodeRegs));
        constexpr int LANES = BLOCKS, KEYS = KT * LANES / kDecoders;         // lanes of a key, one block of features each, and keys of a thread
        const int tid = threadIdx.x % kDecoders, n0 = tid / LANES, kt = tid % LANES;
        const long long block0 = (long long)base * BLOCKS + kt;             // of a slot's first token, in blocks of 16 bytes of codes and a scale
        const int block_pitch = a.n_kv * BLOCKS;
        auto free_phase = [](int j) { return ((uint32_t)(j / kStages) & 1u) ^ 1u; };
        bool ok = true;
        uint4 k_next[KEYS], kc[KEYS]; uint32_t ks_next[KEYS], ks[KEYS];
        auto fetch_k = [&](int j) {
#pragma unroll
            for (int e = 0; e < KEYS; ++e) {
                const long long block = block0 + (long long)token(tile_start(j) + n0 + e * (KT / KEYS)) * block_pitch;
                k_next[e] = load16(a.k_codes + block * 16);
                ks_next[e] = load1(a.k_scales + block);
            }
        };
        auto decode_k = [&](int j) {
            const int s = j % kStages;
            // lanes of the second half of the features take their words in another order, so that a warp's stores spread over the banks
            const int turn = kt & 2;
#pragma unroll
            for (int e = 0; e < KEYS; ++e) {
                kc[e] = turn ? make_uint4(k_next[e].z, k_next[e].w, k_next[e].x, k_next[e].y) : k_next[e];
                ks[e] = ks_next[e];
            }
            if (j + 1 < n_tiles) fetch_k(j + 1);
            if (!tc::mbar_wait(bar_kempty + 8 * s, free_phase(j), &s_abort)) return false;
#pragma unroll
            for (int e = 0; e < KEYS; ++e) {
                const int n = n0 + e * (KT / KEYS);
                const uint32_t sk = tc::smem_u32(sK) + s * K_BYTES + (kt / 2) * (KT * 128) + n * 128;
                const uint32_t f = cache_factor(ks[e]), ff = f | f << 16;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x = i == 0 ? kc[e].x : i == 1 ? kc[e].y : i == 2 ? kc[e].z : kc[e].w;
                    store_chunk(sk + ((((kt & 1) * 4 + (i ^ turn)) ^ (n & 7)) * 16), mul_bf16x2(codes_as_bf16<0>(x), ff), mul_bf16x2(codes_as_bf16<1>(x), ff),
                                mul_bf16x2(codes_as_bf16<2>(x), ff), mul_bf16x2(codes_as_bf16<3>(x), ff));
                }
            }
            fence_async_shared();
            tc::mbar_arrive(bar_kfull + 8 * s);
            return true;
        };
        // Values come as whole blocks too: a thread's own words of eight tokens would be sixteen loads of eight cache lines each (tile of
        // 128 tokens, 128 features: 800 clocks to issue).  Token i of eight ct lies in place 8 i + ct, so that readers' and writers'
        // banks differ.
        constexpr int HALVES = kDecoders / (16 * WORDS);                 // threads of a piece, each with 8 or 4 of the word's features
        const int ct = lane & 7, u = tid / 8, kb = u / (WORDS * HALVES), w0 = u % (WORDS * HALVES) / HALVES, part = u % HALVES;
        uint32_t vs_next[KEYS];
        auto raw = [&](int j, int half, int c, int i) { return tc::smem_u32(sRaw) + (j & 1) * RAW_BYTES + (half * 8 + i) * RAW8 + c * RAW; };
        auto own = [&](int j, int e) { const int n = n0 + e * (KT / KEYS); return raw(j, n / 64, n / 8 % 8, n % 8); };
        auto fetch_v = [&](int j) {
#pragma unroll
            for (int e = 0; e < KEYS; ++e) {
                const long long block = block0 + (long long)token(tile_start(j) + n0 + e * (KT / KEYS)) * block_pitch;
                copy16(own(j, e) + kt * 16, a.v_codes + block * 16);
                vs_next[e] = load1(a.v_scales + block);
            }
            copies_commit();
        };
        auto share_v = [&](int j) {
            copies_wait();
#pragma unroll
            for (int e = 0; e < KEYS; ++e)              // a NaN block counts as zeros: it must not reach the rows that do not see its token
                s_factor[j & 1][kt][n0 + e * (KT / KEYS)] = (uint16_t)(vs_next[e] > mx4::kCacheHi ? 0u : (vs_next[e] + 62) << 7);
            __syncwarp();
            asm volatile("barrier.sync 1, %0;" ::"n"(kDecoders) : "memory");      // (also after a wait that gave up: the others come here)
            if (j + 1 < n_tiles) fetch_v(j + 1);        // (its place was read before tile j was shared)
        };
        auto decode_v = [&](int j) {
            const int s = j % kStages;
            const uint4 factors = *reinterpret_cast<const uint4 *>(&s_factor[j & 1][w0 / 4][kb * 64 + ct * 8]);
            const uint32_t f[4] = {factors.x, factors.y, factors.z, factors.w};
            uint32_t vc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(vc[i]) : "r"(raw(j, kb, ct, i) + w0 * 4) : "memory");
            if (!tc::mbar_wait(bar_vempty + 8 * s, free_phase(j), &s_abort)) return false;
            if (w0 % 4 == 0 && part == 0) {
                uint32_t bad = 0;
                if (((f[0] - 0x00010001u) | (f[1] - 0x00010001u) | (f[2] - 0x00010001u) | (f[3] - 0x00010001u)) & 0x80008000u) {      // some factor is 0
#pragma unroll
                    for (int i = 0; i < 8; ++i) bad |= ((f[i / 2] >> (i & 1) * 16) & 0xFFFFu) == 0u ? 1u << i : 0u;
                    if (bad) s_any_bad = 1;
                }
                s_bad[j & 3][w0 / 4][kb * 8 + ct] = (uint8_t)bad;
            }
            const uint32_t sv = tc::smem_u32(sV) + s * V_BYTES + kb * (DH * 128) + w0 * 8 * 128;
            uint32_t x[4];
            auto feature = [&](auto J, int d) {
                store_chunk(sv + d * 128 + ((ct ^ d) * 16), mul_bf16x2(codes_as_bf16<decltype(J)::value>(x[0]), f[0]), mul_bf16x2(codes_as_bf16<decltype(J)::value>(x[1]), f[1]),
                            mul_bf16x2(codes_as_bf16<decltype(J)::value>(x[2]), f[2]), mul_bf16x2(codes_as_bf16<decltype(J)::value>(x[3]), f[3]));
            };
            auto four = [&](int h) {                    // features 4 h to 4 h + 3 of the word
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = __byte_perm(vc[2 * i], vc[2 * i + 1], h ? 0x7632 : 0x5410);
                feature(std::integral_constant<int, 0>(), 4 * h); feature(std::integral_constant<int, 1>(), 4 * h + 1);
                feature(std::integral_constant<int, 2>(), 4 * h + 2); feature(std::integral_constant<int, 3>(), 4 * h + 3);
            };
            if (HALVES == 1) { four(0); four(1); } else four(part);
            fence_async_shared();
            tc::mbar_arrive(bar_vfull + 8 * s);
            return true;
        };
        if (R::kApart && warp < kDecoders / 32) {
            if (n_tiles > 0) fetch_k(0);
            for (int j = 0; j < n_tiles && ok; ++j) ok = decode_k(j);
        } else if (R::kApart) {
            if (n_tiles > 0) fetch_v(0);
            for (int j = 0; j < n_tiles; ++j) {
                share_v(j);
                ok = ok && decode_v(j);
            }
        } else {
            if (n_tiles > 0) fetch_k(0);
            // Streams over odd and even tiles: keys one tile ahead of values, for the other stream's first scores (128 rows over 1536 tokens,
            // 32 heads: 17.3 us without, 16.7 with); row tiles that share a tile want its values sooner.
            for (int j = PAIR ? 0 : -1; j < n_tiles; ++j) {
                const int jk = PAIR ? j : j + 1;
                if (jk < n_tiles && ok) ok = decode_k(jk);
                if (jk == 0 && n_tiles > 0) fetch_v(0);     // (not sooner: the first keys and the queries come first)
                if (j >= 0) {
                    share_v(j);
                    ok = ok && decode_v(j);
                }
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp) {
        // ---------------- MMA issuer: the whole warp runs the loop with warp-uniform operands, one elected lane issues
        constexpr uint32_t idesc_s = tc::idesc_bf16_f32(QT, KT);
        constexpr uint32_t idesc_o = tc::idesc_bf16_f32(QT, DH);
        const int last = n_streams - 1;
        auto issue_S = [&](int w, int j) {
            const int s = j % kStages;
            if (!__all_sync(0xffffffffu, tc::mbar_wait(bar_kfull + 8 * s, (uint32_t)(j / kStages) & 1u, &s_abort))) return false;
            tc::tc_fence_after();
            const uint32_t sk = tc::smem_u32(sK) + s * K_BYTES, sq = tc::smem_u32(sQ) + (PAIR ? w : 0) * Q_BYTES, d = tmem_S + (uint32_t)(w * KT);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const uint64_t dq = tc::smem_desc_sw128(sq + kb * (QT * 128)), dk = tc::smem_desc_sw128(sk + kb * (KT * 128));
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) tc::mma_bf16_elect(d, dq + (uint64_t)(kk * 2), dk + (uint64_t)(kk * 2), idesc_s, (kb | kk) != 0 ? 1u : 0u);
            }
            tc::mma_commit_elect(bar_s + 8 * w);
            if (!PAIR || w == last) tc::mma_commit_elect(bar_kempty + 8 * s);
            return true;
        };
        bool ok = __all_sync(0xffffffffu, tc::mbar_wait(bar_q, 0, &s_abort));
        for (int w = 0; w < n_streams && ok; ++w) ok = issue_S(w, key_tile(w, 0));
        const int n0 = tiles_of(0);
        for (int i = 0; i < n0 && ok; ++i) {
            for (int w = 0; w < n_streams && ok; ++w) {
                if (i >= tiles_of(w)) continue;
                const int j = key_tile(w, i), s = j % kStages;
                ok = __all_sync(0xffffffffu, tc::mbar_wait(bar_vfull + 8 * s, (uint32_t)(j / kStages) & 1u, &s_abort));
                const uint32_t sv = tc::smem_u32(sV) + s * V_BYTES, tp = tmem_S + (uint32_t)(w * KT), d = tmem_O + (uint32_t)(w * DH);
#pragma unroll
                for (int kb = 0; kb < KT / 64; ++kb) {
                    ok = ok && __all_sync(0xffffffffu, tc::mbar_wait(bar_p + 16 * w + 8 * kb, (uint32_t)i & 1u, &s_abort));
                    if (!ok) break;
                    tc::tc_fence_after();
                    const uint64_t dv = tc::smem_desc_sw128(sv + kb * (DH * 128));
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)          // 16 keys are 8 columns of packed pairs
                        tc::mma_bf16_ts_elect(d, tp + (uint32_t)(kb * 32 + kk * 8), dv + (uint64_t)(kk * 2), idesc_o, (i | kb | kk) != 0 ? 1u : 0u);
                }
                if (!ok) break;
                if (!PAIR || w == last) tc::mma_commit_elect(bar_vempty + 8 * s);
                if (i + 1 < tiles_of(w)) ok = issue_S(w, key_tile(w, i + 1));
                else tc::mma_commit_elect(bar_s + 8 * w);                                   // O of the stream is complete
            }
        }
        __syncwarp();
    } else {
        // ---------------- online softmax, one thread per row, against a reference maximum that follows the true one lazily
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R::kSoftmaxRegs));
        const int w = (warp - kSoftmaxWarp) >> 2, row = (warp & 3) * 32 + lane;
        {
            // in the features' order of a decoded word: (0, 4), (1, 5), (2, 6), (3, 7)
            copies_wait();
#pragma unroll 4
            for (int k = 0; k < BATCH; ++k) {
                const uint32_t at = q_place(q_row + k * ROWS_AT_ONCE);
                uint4 v;
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
                store_chunk(at, __byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
            }
            fence_async_shared();
            tc::mbar_arrive(bar_q);
        }
        const int r = (PAIR ? w * QT : 0) + row;            // row of the CTA
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem_S + (uint32_t)(w * KT) + lane_off, to = tmem_O + (uint32_t)(w * DH) + lane_off;
        const float c = a.scale_log2 * kUnscale;
        const int n_mine = tiles_of(w);
        const int r_lo = s_lo[r] - gap, r_hi = s_hi[r] - gap, r_first = s_first[r];             // (in the sequence without the gap)
        float m = -INFINITY, l = 0.f;                       // reference maximum, denominator (times 2^64)
        uint32_t nan_blocks = 0;
        bool ok = true;
        auto seen64 = [&](int j, int q) {                   // which of 64 keys of tile j the row sees
            const int v0 = tile_start(j) + q * 64;
            return bit_range(r_lo - v0, r_hi - v0) | bit_range(0, r_first - v0);
        };
        auto nan_of = [&](int j) {                          // blocks of features in which the row sees a NaN of tile j
            for (int blk = 0; blk < BLOCKS; ++blk)
                for (int q = 0; q < 2; ++q) {
                    unsigned long long bad = 0;
                    for (int k = 0; k < 8; ++k) bad |= (unsigned long long)s_bad[j & 3][blk][q * 8 + k] << (8 * k);
                    if (bad & seen64(j, q)) nan_blocks |= 1u << blk;
                }
        };
        for (int i = 0; i < n_mine && ok; ++i) {
            ok = tc::mbar_wait(bar_s + 8 * w, (uint32_t)i & 1u, &s_abort);      // (P V of the tile before has finished too)
            if (!ok) break;
            tc::tc_fence_after();
            const int j = key_tile(w, i), v0 = tile_start(j);
            if (i > 0 && *reinterpret_cast<volatile int *>(&s_any_bad)) nan_of(key_tile(w, i - 1));      // its values were decoded by then
            const bool whole = v0 >= r_lo && v0 + KT <= r_hi;
            uint32_t v[64], pk[32];
            auto load = [&](int q) {                        // 64 scores, those of keys that the row does not see -inf
                tc::tmem_ld32(ts + q * 64, v); tc::tmem_ld32(ts + q * 64 + 32, v + 32);
                tc::tmem_ld_wait32(v); tc::tmem_ld_wait32(v + 32);
                if (!whole) {
                    const unsigned long long in = seen64(j, q);
                    const uint32_t in0 = (uint32_t)in, in1 = (uint32_t)(in >> 32);
#pragma unroll
                    for (int k = 0; k < 64; ++k)
                        if (!(((k < 32 ? in0 : in1) >> (k & 31)) & 1u)) v[k] = 0xFF800000u;
                }
            };
            auto row_max = [&]() {
                float mx[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = __uint_as_float(v[k]);
#pragma unroll
                for (int k = 4; k + 7 < 64; k += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx[e] = tc::max3(mx[e], __uint_as_float(v[k + e]), __uint_as_float(v[k + 4 + e]));
#pragma unroll
                for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], __uint_as_float(v[60 + e]));
                return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
            };
            unsigned long long sum2[2];
            auto half = [&]() {                             // 64 keys: 32 columns of packed pairs
                const float mc = m == -INFINITY ? 0.f : 64.f - m * c;
                const unsigned long long c2 = tc::pack_f32x2(c, c), mc2 = tc::pack_f32x2(mc, mc);
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    float e0, e1;
                    tc::unpack_f32x2(tc::fma_f32x2(tc::pack_f32x2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), c2, mc2), e0, e1);
                    const float p0 = tc::ex2_approx(e0), p1 = tc::ex2_approx(e1);
                    sum2[k & 1] = tc::add_f32x2(sum2[k & 1], tc::pack_f32x2(p0, p1));
                    __nv_bfloat162 hh = __floats2bfloat162_rn(p0, p1);
                    pk[k] = *reinterpret_cast<uint32_t *>(&hh);
                }
            };
            auto hand = [&](int q) {
                tc::tmem_st32(ts + q * 32, pk);
                tc::tmem_st_wait();
                tc::tc_fence_before();                      // S has been read, this half of P written, O rescaled
                tc::mbar_arrive(bar_p + 16 * w + 8 * q);
            };
            load(1);
            const float m_hi = row_max();
            load(0);
            sum2[0] = sum2[1] = 0ull;
            const float m_row = fmaxf(row_max(), m_hi);
            if (i == 0) {
                m = m_row;
            } else {
                const bool move = (m_row - m) * c > kLazy;
                if (__any_sync(0xffffffffu, move)) {
                    const float alpha = move ? tc::ex2_approx((m - m_row) * c) : 1.0f;
#pragma unroll 1
                    for (int q = 0; q < DH / 32; ++q) {
                        uint32_t o[32];
                        tc::tmem_ld32(to + q * 32, o);
                        tc::tmem_ld_wait32(o);
#pragma unroll
                        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                        tc::tmem_st32(to + q * 32, o);
                    }
                    if (move) { l *= alpha; m = m_row; }
                }
            }
            half();
            hand(0);
            load(1);
            half();
            hand(1);
            float s0, s1;
            tc::unpack_f32x2(tc::add_f32x2(sum2[0], sum2[1]), s0, s1);
            l += s0 + s1;
        }
        if (n_mine > 0) {
            ok = ok && tc::mbar_wait(bar_s + 8 * w, (uint32_t)n_mine & 1u, &s_abort);       // the last P V
            if (ok && *reinterpret_cast<volatile int *>(&s_any_bad)) nan_of(key_tile(w, n_mine - 1));
        } else if (PAIR) {
            // Outputs pass through the queries' place below.  A stream with tiles has seen its products, which wait for all queries; this one has
            // waited for nothing, and every softmax warp puts rows into every warp's part (24 x 256 rows, 32 heads, one sequence with keys:
            // one zero in 1300 was a piece of a query).
            ok = tc::mbar_wait(bar_q, 0, &s_abort);
        }
        // output columns of this thread, and the factors of the streams' accumulators
        constexpr int COLS = PAIR ? DH : DH / 2;
        const int col0 = PAIR ? 0 : w * COLS;
        float f0 = 0.f, f1 = 0.f;                           // PAIR: f0 of the own stream
        bool write = ok && !s_abort;
        if (PAIR) {
            f0 = inverse(r, l);
        } else {
            s_max[w][row] = m; s_den[w][row] = l; s_nan[w][row] = nan_blocks;
            tc::tc_fence_before();
            tc::mbar_arrive(bar_x);
            write = tc::mbar_wait(bar_x, 0, &s_abort) && write && !s_abort;
            const float m0 = s_max[0][row], m1 = s_max[1][row], mm = fmaxf(m0, m1);
            f0 = m0 == -INFINITY ? 0.f : tc::ex2_approx((m0 - mm) * c); f1 = m1 == -INFINITY ? 0.f : tc::ex2_approx((m1 - mm) * c);
            const float den = f0 * s_den[0][row] + f1 * s_den[1][row];
            nan_blocks = s_nan[0][row] | s_nan[1][row];
            if (splits == 1) {
                const float inv = inverse(row, den);
                f0 *= inv; f1 *= inv;
            } else if (w == 0) s_ml[row] = make_float2(mm, den);
        }
        if (__all_sync(0xffffffffu, write)) {
            tc::tc_fence_after();
            const uint32_t t0 = tmem_O + lane_off + (uint32_t)(PAIR ? w * DH : col0);
            // the rows' outputs pass through the queries' place, so that a row leaves in whole lines; 16-byte chunks rotated by the row
            constexpr int CH = COLS / 8, TURN = CH < 8 ? CH - 1 : 7;
            const uint32_t park = tc::smem_u32(sQ) + (PAIR ? w * Q_BYTES : w * (QT * COLS * 2)) + (warp & 3) * 32 * COLS * 2;
            auto place = [&](int rr, int chunk) { return park + rr * (COLS * 2) + ((chunk ^ ((CH < 8 ? rr >> 1 : rr) & TURN)) * 16); };
#pragma unroll
            for (int q = 0; q < COLS / 32; ++q) {
                uint32_t o[32], o1[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) o[k] = o1[k] = 0u;
                if (PAIR ? n_mine > 0 : n_streams > 0) { tc::tmem_ld32(t0 + q * 32, o); tc::tmem_ld_wait32(o); }
                if (!PAIR && n_streams > 1) { tc::tmem_ld32(t0 + DH + q * 32, o1); tc::tmem_ld_wait32(o1); }
                const bool nan = (nan_blocks >> (col0 / 32 + q)) & 1u;
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    float x = __uint_as_float(o[k]) * f0;
                    if (!PAIR) x = fmaf(__uint_as_float(o1[k]), f1, x);
                    o[k] = nan ? 0x7FC00000u : __float_as_uint(x);
                }
                if (!PAIR && splits > 1) {
                    // rotated by the row, so that a warp's stores spread over the banks
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        store_chunk(s_o + row * (DH * 4) + ((col0 / 4 + q * 8 + i + row) % (DH / 4)) * 16, o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t wd[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            __nv_bfloat162 hh = __floats2bfloat162_rn(__uint_as_float(o[8 * i + 2 * t]), __uint_as_float(o[8 * i + 2 * t + 1]));
                            wd[t] = *reinterpret_cast<uint32_t *>(&hh);
                        }
                        store_chunk(place(lane, q * 4 + i), wd[0], wd[1], wd[2], wd[3]);
                    }
                }
            }
            if (PAIR || splits == 1) {
                __syncwarp();
                constexpr int AT_ONCE = 32 / CH;            // rows of a warp's store
#pragma unroll 4
                for (int rr = lane / CH; rr < 32; rr += AT_ONCE) {
                    const int rg = (PAIR ? w * QT : 0) + (warp & 3) * 32 + rr;
                    if (rg >= n_rows || s_first[rg] < 0) continue;
                    uint4 v;
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(place(rr, lane % CH)) : "memory");
                    *reinterpret_cast<uint4 *>(a.out + row_of(rg, a.ld_out) + col0 + lane % CH * 8) = v;
                }
            }
        }
    }
    if (!PAIR && splits > 1) {
        // ---------------- join the ranks: each fetches its share of the rows from all of them, whole rows to a warp (pushed by the threads
        // that have the rows, 16 bytes to each, they took 5500 clocks: 128 rows over 1536 tokens 15.2 us, 14.15 so)
        tc::cluster_sync();
        if (!s_abort) {
            for (int x = threadIdx.x; x < share * (DH / 4); x += kThreads) {
                const int row = rank * share + x / (DH / 4), col = x % (DH / 4);
                if (row >= n_rows || s_first[row] < 0) continue;
                const uint32_t ml_at = tc::smem_u32(&s_ml[row]), o_at = s_o + row * (DH * 4) + (col + row) % (DH / 4) * 16;
                float M = -INFINITY, L = 0.f;
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f), o[8];
                float2 ml[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    ml[k] = k < splits ? load_remote2(tc::mapa(ml_at, (uint32_t)k)) : make_float2(-INFINITY, 0.f);
                    o[k] = k < splits ? load_remote4(tc::mapa(o_at, (uint32_t)k)) : sum;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) M = fmaxf(M, ml[k].x);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float f = ml[k].x == -INFINITY ? 0.f : tc::ex2_approx((ml[k].x - M) * (a.scale_log2 * kUnscale));
                    L += f * ml[k].y;
                    sum.x += f * o[k].x; sum.y += f * o[k].y; sum.z += f * o[k].z; sum.w += f * o[k].w;
                }
                const float inv = inverse(row, L);
                const __nv_bfloat162 x0 = __floats2bfloat162_rn(sum.x * inv, sum.y * inv), x1 = __floats2bfloat162_rn(sum.z * inv, sum.w * inv);
                *reinterpret_cast<uint2 *>(a.out + row_of(row, a.ld_out) + col * 4) =
                    make_uint2(*reinterpret_cast<const uint32_t *>(&x0), *reinterpret_cast<const uint32_t *>(&x1));
            }
        }
        tc::cluster_sync();                                 // a rank's output stays until the others have read it
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) { tc::tc_fence_after(); tc::tmem_dealloc(tmem_base, TMEM_COLS); }
    if (threadIdx.x == 0 && s_abort && a.err) atomicExch(a.err, SFS_ERR_TIMEOUT);
}

template <int DH, bool PAIR>
int32_t launch(const Cache4Args &a, int log_splits, cudaStream_t stream)
{
    using R = Roles<DH, PAIR>;
    constexpr int NQ = PAIR ? 2 : 1;
    constexpr size_t shared = 1024 + (size_t)NQ * QT * DH * 2 + (size_t)kStages * 2 * KT * DH * 2 + 2 * (size_t)(KT / 8) * (8 * (DH / 2 + 16) + DH / 2) + kBars * 8 + 16;
    const long long row_tiles = ((long long)a.n_q * a.group + NQ * QT - 1) / (NQ * QT), ctas = ((long long)a.batch * a.n_kv * row_tiles) << log_splits;
    SFS_REQUIRE(ctas <= 0x7FFFFFFF, SFS_ERR_UNSUPPORTED, "attention_cache4: too many rows and heads for one call");
    SFS_CUDA(allow_shared(attention_cache4_many_kernel<DH, PAIR>, shared));
    // the softmax warps wait for registers that the launch must have brought: without them the kernel would not end
    cudaFuncAttributes attr;
    SFS_CUDA(cudaFuncGetAttributes(&attr, attention_cache4_many_kernel<DH, PAIR>));
    SFS_REQUIRE(attr.numRegs >= R::kRegs, SFS_ERR_UNSUPPORTED, "attention_cache4: built with %d registers a thread, %d needed", attr.numRegs, R::kRegs);
    if (log_splits > 0) SFS_CUDA(launch_pdl_cluster(attention_cache4_many_kernel<DH, PAIR>, 1 << log_splits, dim3((unsigned)ctas), dim3(R::kThreads), shared, stream, a, log_splits, (int)row_tiles));
    else SFS_CUDA(launch_pdl(attention_cache4_many_kernel<DH, PAIR>, dim3((unsigned)ctas), dim3(R::kThreads), shared, stream, a, 0, (int)row_tiles));
    return SFS_OK;
}

// Row tiles in pairs, or alone: up to one wave of CTAs then, two key tiles for each.  Clusters do not cover every SM, since they do not
// cross the GPU's partitions: 128 CTAs in clusters of four run at once, in clusters of eight they do not (128 rows over 1536 tokens, 16
// heads: 14.6 us with four, 25.4 with eight).
// Microseconds: 5.5 for a CTA's start and end, 2.5 for a join, and for a key tile 1.95 of 128 features or 1.35 of 64 (72 rows over 5344
// tokens, 4 x 32 heads: 87 and 61), 2.55 and 2.0 for a pair's (2048 rows over 2048, 32 heads: 94; over 8192, 2 x 32 heads of 64: 523).
// So 544 rows over 1692 tokens of 32 heads go in 96 pairs, 46 us, and not in two rounds of 160 CTAs, 62.6 when pairs took 48.
struct Many { bool pair; int log_splits; double us; };
Many plan(const Cache4Args &a, int64_t tokens, int head_dim)
{
    const long long row_tiles = ((long long)a.n_q * a.group + QT - 1) / QT, heads = (long long)a.batch * a.n_kv, sms = gemm_num_sms();
    const long long tiles = (tokens + KT - 1) / KT, pairs = heads * ((row_tiles + 1) / 2), singles = heads * row_tiles;
    int log_splits = 0;
    while (log_splits < 3 && (singles << (log_splits + 1)) <= (log_splits == 2 ? sms / 2 : sms * 7 / 8) && tokens > (2 * KT) << log_splits) ++log_splits;
    const Many one = {false, log_splits, (double)(((singles << log_splits) + sms - 1) / sms) * (5.5 + (head_dim == 128 ? 1.95 : 1.35) * (double)((tiles + (1 << log_splits) - 1) >> log_splits)) + (log_splits > 0 ? 2.5 : 0.0)};
    const Many two = {true, 0, (double)((pairs + sms - 1) / sms) * (5.5 + (head_dim == 128 ? 2.55 : 2.0) * (double)tiles)};
    return row_tiles > 1 && two.us < one.us ? two : one;
}

}  // namespace

double attention_cache4_many_us(const Cache4Args &a, int64_t tokens, int head_dim) { return plan(a, tokens, head_dim).us; }

int32_t attention_cache4_many(const Cache4Args &a, int64_t tokens, int head_dim, cudaStream_t stream)
{
    const Many p = plan(a, tokens, head_dim);
    if (p.pair) return head_dim == 128 ? launch<128, true>(a, 0, stream) : launch<64, true>(a, 0, stream);
    return head_dim == 128 ? launch<128, false>(a, p.log_splits, stream) : launch<64, false>(a, p.log_splits, stream);
}

}  // namespace sfs

// Quantisation of matrices and of a key / value cache to microscaled 4-bit numbers, and the values they stand for.
//
// A half-warp takes 128 consecutive values of a row, four blocks of 32: a lane holds 8 of them (16 bytes of bf16), a block's largest
// magnitude is the maximum of the bit patterns over 4 lanes, so a NaN or an infinity shows in it, and each value is scaled by a power of
// two (exact) and rounded once, by the conversion instruction.  A warp works on 256 to 1024 neighbouring columns (see pieces), so that addresses
// are computed once for up to four loads in flight: with one piece at a time, found anew, the instructions and not the memory set the pace
// (126464 x 4096 to codes and back: 624 us, 483 so; 2.6 GB move, 5.4 TB/s of a measured copy rate of 6.57).  Rows of at most 256 columns go
// several to a warp, rows off 16-byte boundaries by words that shifts put together.
#include "attention_cache4.cuh"
#include "gemm.cuh"
#include <algorithm>

namespace sfs {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// Eight values of a row from column `col` on, zeros behind the last column; as they lie in memory, so that several loads can be in flight.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *at) { a = __ldcs(reinterpret_cast<const uint4 *>(at)); }
    __device__ __forceinline__ void load_some(const __nv_bfloat16 *at, int n)
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i < n ? (uint32_t)__bfloat16_as_ushort(at[i]) : 0u;
        a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
    // bits of the largest magnitude as a float's; bit patterns of bf16 magnitudes are in order, NaN and infinity on top
    __device__ __forceinline__ uint32_t largest() const
    {
        const uint32_t m = __vmaxu2(__vmaxu2(a.x & 0x7FFF7FFFu, a.y & 0x7FFF7FFFu), __vmaxu2(a.z & 0x7FFF7FFFu, a.w & 0x7FFF7FFFu));
        return max(m & 0xFFFF0000u, m << 16);
    }
    __device__ __forceinline__ void get(float *v) const
    {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
    }
};
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float *at) { a = __ldcs(reinterpret_cast<const float4 *>(at)); b = __ldcs(reinterpret_cast<const float4 *>(at) + 1); }
    __device__ __forceinline__ void load_some(const float *at, int n)
    {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? at[i] : 0.f;
        a = make_float4(v[0], v[1], v[2], v[3]); b = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ uint32_t largest() const
    {
        float v[8];
        get(v);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        return m;
    }
    __device__ __forceinline__ void get(float *v) const { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w; }
};
// eight bf16 values to a row of T, n of them at a place that takes no wide store
__device__ __forceinline__ void put(__nv_bfloat16 *at, const uint4 &v) { *reinterpret_cast<uint4 *>(at) = v; }
__device__ __forceinline__ void put(float *at, const uint4 &v)
{
    reinterpret_cast<float4 *>(at)[0] = make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u));
    reinterpret_cast<float4 *>(at)[1] = make_float4(__uint_as_float(v.z << 16), __uint_as_float(v.z & 0xFFFF0000u), __uint_as_float(v.w << 16), __uint_as_float(v.w & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ void put_some(T *at, const uint4 &v, int n)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            const uint32_t h = (i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
            if constexpr (sizeof(T) == 4) at[i] = __uint_as_float(h << 16); else at[i] = __ushort_as_bfloat16((unsigned short)h);
        }
}

// ---- rows that do not lie on 16-byte boundaries: a warp's bytes are consecutive, so lanes load and store the aligned vectors that hold them
// and shift their own bytes out of two neighbours' (element by element, 103658 x 3706 to codes and back took 1519 us).

// words `at` .. `at` + N - 1 of w, where a word may start in the middle of another: `at` in bytes, even, below 16
template <int N>
__device__ __forceinline__ void words_at(const uint32_t (&w)[N + 4], uint32_t at, uint32_t (&out)[N])
{
    uint32_t x[N + 4];
#pragma unroll
    for (int i = 0; i < N + 4; ++i) x[i] = (at & 8) && i + 2 < N + 4 ? w[i + 2 < N + 4 ? i + 2 : i] : w[i];
#pragma unroll
    for (int i = 0; i + 1 < N + 4; ++i) x[i] = (at & 4) ? x[i + 1] : x[i];
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = (at & 2) ? __funnelshift_r(x[i], x[i + 1], 16) : x[i];
}
// the aligned vector at `at`, of which only what lies in [lo, hi) is read
__device__ __forceinline__ uint4 load_within(uintptr_t at, uintptr_t lo, uintptr_t hi)
{
    if (at >= lo && at + 16 <= hi) return __ldcs(reinterpret_cast<const uint4 *>(at));
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (at + 2 * i >= lo && at + 2 * i < hi) w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t *>(at + 2 * i) << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// What lane + 1 has, and lane 31 what lane 0 has of the warp's next piece, or `last` behind the last one.
__device__ __forceinline__ uint4 of_next_lane(const uint4 &mine, const uint4 &piece_after, const uint4 &last, bool is_last, int lane)
{
    const uint4 t = lane == 0 && !is_last ? piece_after : mine;
    uint4 n;
    n.x = __shfl_sync(0xffffffffu, t.x, (lane + 1) & 31); n.y = __shfl_sync(0xffffffffu, t.y, (lane + 1) & 31);
    n.z = __shfl_sync(0xffffffffu, t.z, (lane + 1) & 31); n.w = __shfl_sync(0xffffffffu, t.w, (lane + 1) & 31);
    return lane == 31 && is_last ? last : n;
}
// What lane - 1 has, and lane 0 what lane 31 had of the piece before.
__device__ __forceinline__ uint4 of_lane_before(const uint4 &mine, const uint4 &piece_before, int lane)
{
    const uint4 t = lane == 31 ? piece_before : mine;
    uint4 n;
    n.x = __shfl_sync(0xffffffffu, t.x, (lane + 31) & 31); n.y = __shfl_sync(0xffffffffu, t.y, (lane + 31) & 31);
    n.z = __shfl_sync(0xffffffffu, t.z, (lane + 31) & 31); n.w = __shfl_sync(0xffffffffu, t.w, (lane + 31) & 31);
    return n;
}
// a warp's U pieces of a row, lane's first value at `p`, the row's end at `row_end`, the matrix from `lo` to `hi`
template <int U>
__device__ __forceinline__ void load_shifted(Eight<__nv_bfloat16> (&v)[U], uintptr_t p, uintptr_t row_end, uintptr_t lo, uintptr_t hi, int)
{
    // five aligned words hold a lane's eight values (fewer instructions than vectors and shuffles, and the cache serves them as fast)
    const uint32_t shift = (uint32_t)(p & 2) * 8;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uintptr_t at = (p & ~(uintptr_t)3) + u * 512;
        if (p + u * 512 + 16 <= row_end && at >= lo && at + 20 <= hi) {
            uint32_t w[5];
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = __ldg(reinterpret_cast<const uint32_t *>(at) + i);
            v[u].a = make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift), __funnelshift_r(w[2], w[3], shift), __funnelshift_r(w[3], w[4], shift));
        } else if (p + u * 512 < row_end) v[u].load_some(reinterpret_cast<const __nv_bfloat16 *>(p + u * 512), (int)min((uintptr_t)8, (row_end - p - u * 512) / 2));
        else v[u].zero();
    }
}
template <int U>
__device__ __forceinline__ void load_shifted(Eight<float> (&v)[U], uintptr_t p, uintptr_t row_end, uintptr_t lo, uintptr_t hi, int lane)
{
    const uint32_t m = (uint32_t)(p & 15);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    uint4 a[U], b[U], last = zero;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uintptr_t at = p - m + u * 1024;
        a[u] = at < row_end ? load_within(at, lo, hi) : zero;
        b[u] = at + 16 < row_end ? load_within(at + 16, lo, hi) : zero;
    }
    if (lane == 31 && m != 0) { const uintptr_t at = p - m + (U - 1) * 1024 + 32; if (at < row_end) last = load_within(at, lo, hi); }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint4 n = of_next_lane(a[u], a[u + 1 < U ? u + 1 : u], last, u + 1 == U, lane);
        const uint32_t w[12] = {a[u].x, a[u].y, a[u].z, a[u].w, b[u].x, b[u].y, b[u].z, b[u].w, n.x, n.y, n.z, n.w};
        uint32_t x[8];
        words_at<8>(w, m, x);
        const int left = (int)min((long long)8, max(0ll, ((long long)row_end - (long long)(p + u * 1024)) / 4));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i >= left ? 0u : x[i];
        v[u].a = make_float4(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3]));
        v[u].b = make_float4(__uint_as_float(x[4]), __uint_as_float(x[5]), __uint_as_float(x[6]), __uint_as_float(x[7]));
    }
}
// The reverse: piece u of a warp's run [lo, hi) of a row, `v` this lane's values at `p`, `before` its piece u - 1.  Whole vectors inside the
// run are stored by the lane in whose place they begin, what is left at the run's ends element by element.
template <typename T>
__device__ __forceinline__ void store_shifted(uintptr_t p, uintptr_t lo, uintptr_t hi, const uint4 &v, const uint4 &before, int lane)
{
    constexpr int WORDS = sizeof(T) == 4 ? 8 : 4;
    const uint32_t m = (uint32_t)(p & 15);
    const uint4 b = of_lane_before(v, before, lane);
    uint32_t w[WORDS + 4], x[WORDS];
    if constexpr (sizeof(T) == 4) {                         // (a bf16 value is the upper half of an fp32 one)
        const uint32_t t[12] = {b.z << 16, b.z & 0xFFFF0000u, b.w << 16, b.w & 0xFFFF0000u, v.x << 16, v.x & 0xFFFF0000u, v.y << 16, v.y & 0xFFFF0000u,
                                v.z << 16, v.z & 0xFFFF0000u, v.w << 16, v.w & 0xFFFF0000u};
#pragma unroll
        for (int i = 0; i < 12; ++i) w[i] = t[i];
    } else {
        const uint32_t t[8] = {b.x, b.y, b.z, b.w, v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = t[i];
    }
    if (m == 0) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) x[i] = w[i + 4];
    } else words_at<WORDS>(w, 16 - m, x);
    const uintptr_t a = p - m, own_end = p + WORDS * 4;
#pragma unroll
    for (int i = 0; i < WORDS / 4; ++i)
        if (a + 16 * i >= lo && a + 16 * i + 16 <= hi) *reinterpret_cast<uint4 *>(a + 16 * i) = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    if (a < lo || ((own_end + 15) & ~(uintptr_t)15) > hi) { // this lane has values that no whole vector holds
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uintptr_t q = p + e * sizeof(T), qa = q & ~(uintptr_t)15;
            if (q < hi && !(qa >= lo && qa + 16 <= hi)) {
                if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t *>(q) = w[4 + e];
                else *reinterpret_cast<uint16_t *>(q) = (uint16_t)((e & 1) ? w[4 + e / 2] >> 16 : w[4 + e / 2]);
            }
        }
    }
}

// the four lanes of a block: its scale, and this lane's eight codes
template <typename T>
__device__ __forceinline__ uint32_t quantize8(const Eight<T> &x, int lo, int hi, int &c)
{
    uint32_t a = x.largest();
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
    c = mx4::scale_of(a, lo, hi);
    const float f = mx4::inverse_scale(c);
    float v[8];
    x.get(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= f;
    const uint32_t w = mx4::encode8(v);
    return c == 255 ? 0u : w;
}

// where the four scale bytes of a row's blocks 4 q .. 4 q + 3 lie in a matrix's tiles
__device__ __forceinline__ size_t scale_quad(int row, int q, int quads) { return ((size_t)(row >> 7) * quads + q) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4; }

// A warp's position, a segment of a row, and the step to its next one without a division.  A segment is 2 U quads: half-warp h takes
// the quads h, h + 2, ..., so that a warp's loads are 512 consecutive bytes.
struct Walk {
    int row, seg, step_rows, step_segs, segs;
    __device__ __forceinline__ Walk(int first, int stride, int segs_) : segs(segs_)
    {
        row = first / segs; seg = first - row * segs;
        step_rows = stride / segs; step_segs = stride - step_rows * segs;
    }
    __device__ __forceinline__ void next() { row += step_rows; seg += step_segs; if (seg >= segs) { seg -= segs; ++row; } }
};
__device__ __forceinline__ Walk warps_of_grid(int segs) { return Walk(blockIdx.x * kWarps + threadIdx.x / 32, gridDim.x * kWarps, segs); }

template <typename T, int U, bool WIDE>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const T *__restrict__ x, long long ldx, int rows, int cols, uint8_t *__restrict__ codes, long long ld_codes,
                uint8_t *__restrict__ scales, int quads)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15, tile_rows = (rows + 127) / 128 * 128, blocks = (cols + 31) / 32;
    for (Walk at = warps_of_grid((quads + 2 * U - 1) / (2 * U)); at.row < tile_rows; at.next()) {
        const int quad0 = at.seg * 2 * U + half, col0 = quad0 * 128 + l * 8;
        const bool in = at.row < rows, full = in && WIDE && (at.seg + 1) * 2 * U * 128 <= cols;
        const T *src = x + at.row * ldx + col0;
        Eight<T> v[U];
        if (WIDE || !in) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int left = cols - col0 - u * 256;
                if (full || (in && left >= 8)) v[u].load(src + u * 256);
                else if (in && left > 0) v[u].load_some(src + u * 256, left);
                else v[u].zero();
            }
        } else
            load_shifted<U>(v, (uintptr_t)src, (uintptr_t)(x + at.row * ldx + cols), (uintptr_t)x, (uintptr_t)(x + (rows - 1) * ldx + cols), lane);
        uint8_t *to = codes + at.row * ld_codes + quad0 * 64 + l * 4, *s = scales + scale_quad(at.row, quad0, quads) + (l >> 2);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            int c;
            const uint32_t w = quantize8(v[u], 0, 254, c);
            const bool block_in = full || (in && (quad0 + 2 * u) * 4 + (l >> 2) < blocks);
            if (block_in) *reinterpret_cast<uint32_t *>(to + u * 128) = w;
            if ((l & 3) == 0 && quad0 + 2 * u < quads) s[u * 1024] = block_in ? (uint8_t)c : (uint8_t)0;      // the padding of the tiles holds zeros
        }
    }
}

template <typename T, int U, bool WIDE>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t *__restrict__ codes, long long ld_codes, const uint8_t *__restrict__ scales, int rows, int cols, T *__restrict__ x,
                  long long ldx, int quads)
{
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15;
    for (Walk at = warps_of_grid((quads + 2 * U - 1) / (2 * U)); at.row < rows; at.next()) {
        const int quad0 = at.seg * 2 * U + half, col0 = quad0 * 128 + l * 8;
        const uint8_t *from = codes + at.row * ld_codes + quad0 * 64 + l * 4, *s = scales + scale_quad(at.row, quad0, quads) + (l >> 2);
        uint32_t w[U], c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            w[u] = c[u] = 0;
            if (col0 + u * 256 < cols) { w[u] = __ldcs(reinterpret_cast<const uint32_t *>(from + u * 128)); c[u] = s[u * 1024]; }
        }
        T *to = x + at.row * ldx + col0;
        if (WIDE) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int left = cols - col0 - u * 256;
                const uint4 v = mx4::decode8(w[u], c[u]);
                if (left >= 8) put(to + u * 256, v); else put_some(to + u * 256, v, left);
            }
        } else {
            const uintptr_t lo = (uintptr_t)(x + at.row * ldx + at.seg * 2 * U * 128), hi = min(lo + 2 * U * 128 * sizeof(T), (uintptr_t)(x + at.row * ldx + cols));
            uint4 before = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint4 v = mx4::decode8(w[u], c[u]);
                store_shifted<T>((uintptr_t)(to + u * 256), lo, hi, v, before, lane);
                before = v;
            }
        }
    }
}

// Rows of at most 256 columns: LANES lanes for one, so that a warp works on 32 / LANES rows (131072 x 32 with a warp for a row: 47 us).
template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads)
quantize_short_kernel(const T *__restrict__ x, long long ldx, int rows, int cols, uint8_t *__restrict__ codes, long long ld_codes, uint8_t *__restrict__ scales, int wide)
{
    pdl_wait();
    pdl_trigger();
    constexpr int PER = 32 / LANES, U = 4, QUADS = LANES == 32 ? 2 : 1;
    const int lane = threadIdx.x & 31, l = lane % LANES, col = l * 8, tile_rows = (rows + 127) / 128 * 128, stride = gridDim.x * kWarps * PER;
    for (int row0 = (blockIdx.x * kWarps + threadIdx.x / 32) * PER + lane / LANES; __any_sync(0xffffffffu, row0 < tile_rows); row0 += U * stride) {
        Eight<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * stride;
            const T *src = x + row * ldx + col;
            if (row >= rows || col >= cols) v[u].zero();
            else if (wide && col + 8 <= cols) v[u].load(src);
            else v[u].load_some(src, cols - col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * stride;
            int c;
            const uint32_t w = quantize8(v[u], 0, 254, c);
            const bool in = row < rows && (l & ~3) * 8 < cols;                    // the lane's block exists
            if (in) *reinterpret_cast<uint32_t *>(codes + row * ld_codes + l * 4) = w;
            uint32_t s = in ? (uint32_t)c << ((l & 12) * 2) : 0u;                  // the padding of the tiles holds zeros
            if (LANES >= 8) s |= __shfl_xor_sync(0xffffffffu, s, 4);
            if (LANES >= 16) s |= __shfl_xor_sync(0xffffffffu, s, 8);
            if ((l & 15) == 0 && row < tile_rows) *reinterpret_cast<uint32_t *>(scales + scale_quad(row, l / 16, QUADS)) = s;
        }
    }
}
template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads)
dequantize_short_kernel(const uint8_t *__restrict__ codes, long long ld_codes, const uint8_t *__restrict__ scales, int rows, int cols, T *__restrict__ x, long long ldx, int wide)
{
    pdl_wait();
    pdl_trigger();
    constexpr int PER = 32 / LANES, U = 4, QUADS = LANES == 32 ? 2 : 1;
    const int lane = threadIdx.x & 31, l = lane % LANES, col = l * 8, stride = gridDim.x * kWarps * PER;
    if (col >= cols) return;
    for (int row0 = (blockIdx.x * kWarps + threadIdx.x / 32) * PER + lane / LANES; row0 < rows; row0 += U * stride) {
        uint32_t w[U], c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * stride;
            w[u] = c[u] = 0;
            if (row < rows) { w[u] = *reinterpret_cast<const uint32_t *>(codes + row * ld_codes + l * 4); c[u] = scales[scale_quad(row, l / 16, QUADS) + ((l & 15) >> 2)]; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * stride;
            if (row >= rows) break;
            const uint4 v = mx4::decode8(w[u], c[u]);
            if (wide && col + 8 <= cols) put(x + row * ldx + col, v); else put_some(x + row * ldx + col, v, cols - col);
        }
    }
}

// ---- the cache: a token's keys (or values) of all heads are one row of blocks, codes and scales each in one run of bytes ------------

constexpr int kStoreRows = 8;                               // tokens of a CTA, at most

// a warp's segment of one token's keys or values, `from` its row, into the cache at `slot`
template <typename T, int U>
__device__ __forceinline__ void store_segment(const T *from, bool wide, int slot, int seg, uint8_t *codes, uint8_t *scales, int width)
{
    const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15, blocks = width / 32;
    const int quad0 = seg * 2 * U + half, col0 = quad0 * 128 + l * 8;
    Eight<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (col0 + u * 256 >= width) x[u].zero();           // (a width is whole blocks: eight values are in or out together)
        else if (wide) x[u].load(from + col0 + u * 256);
        else x[u].load_some(from + col0 + u * 256, 8);
    }
    uint8_t *to = codes + (size_t)slot * (width / 2) + quad0 * 64 + l * 4, *s = scales + (size_t)slot * blocks + quad0 * 4 + (l >> 2);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        int c;
        const uint32_t w = quantize8(x[u], mx4::kCacheLo, mx4::kCacheHi, c);
        if (col0 + u * 256 < width) {
            *reinterpret_cast<uint32_t *>(to + u * 128) = w;
            if ((l & 3) == 0) s[u * 8] = (uint8_t)c;
        }
    }
}

template <typename T, int U>
__global__ void __launch_bounds__(kThreads)
cache_store_kernel(uint8_t *__restrict__ k_codes, uint8_t *__restrict__ k_scales, uint8_t *__restrict__ v_codes, uint8_t *__restrict__ v_scales,
                   int n_slots, int width, const T *__restrict__ k, long long ld_k, const T *__restrict__ v, long long ld_v, int wide_k, int wide_v,
                   const int32_t *__restrict__ slots, int n_rows, int cta_rows)
{
    pdl_wait();
    pdl_trigger();
    __shared__ int s_slot[kStoreRows];
    const int r0 = blockIdx.x * cta_rows;
    if (threadIdx.x < kStoreRows) {
        const int r = r0 + threadIdx.x;
        const int slot = r < n_rows && (int)threadIdx.x < cta_rows ? (slots ? slots[r] : r) : -1;
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
    for (Walk at(threadIdx.x / 32, kWarps, ((width + 127) / 128 + 2 * U - 1) / (2 * U)); at.row < cta_rows; at.next()) {
        const int slot = s_slot[at.row];
        if (slot >= 0)                                      // (a warp works on one row)
            store_segment<T, U>(src + (r0 + at.row) * ld, keys ? wide_k : wide_v, slot, at.seg, keys ? k_codes : v_codes, keys ? k_scales : v_scales, width);
    }
}

// Many rows with slots of their own.  Which of several rows with one slot is the last is found by looking at all later slots, so the work grows
// with the square of the rows over the rows of a CTA: here up to 1024, keys and values together, whose slots lie in a table in shared memory
// (open addressing, at most a quarter of it taken), where a later slot is mostly looked up in one or two reads.  262144 rows of 8 heads of 128:
// 378 us, 267 without slots, 207 of bytes; 1048576: 2145, 828 of bytes, the rest lookups.
constexpr int kManyRows = 1024, kManyThreads = 512;
constexpr int kTableBits = 12, kTable = 1 << kTableBits;
static_assert(kTable >= 4 * kManyRows, "a quarter");

template <typename T, int U>
__global__ void __launch_bounds__(kManyThreads, 2)
cache_store_many_kernel(uint8_t *__restrict__ k_codes, uint8_t *__restrict__ k_scales, uint8_t *__restrict__ v_codes, uint8_t *__restrict__ v_scales,
                        int n_slots, int width, const T *__restrict__ k, long long ld_k, const T *__restrict__ v, long long ld_v, int wide_k, int wide_v,
                        const int32_t *__restrict__ slots, int n_rows, int cta_rows)
{
    pdl_wait();
    pdl_trigger();
    __shared__ int s_key[kTable], s_last[kTable];           // a slot, and the last of this CTA's rows that names it
    __shared__ int s_slot[kManyRows];                       // a row's place in the table, then its slot, or -1 for a row that is left out
    const int r0 = blockIdx.x * cta_rows, rows = min(cta_rows, n_rows - r0);
    auto place = [](int slot) { return ((uint32_t)slot * 2654435769u) >> (32 - kTableBits); };
    for (int i = threadIdx.x; i < kTable; i += kManyThreads) s_key[i] = s_last[i] = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < rows; i += kManyThreads) {
        const int slot = slots[r0 + i];
        int at = -1;
        if ((unsigned)slot < (unsigned)n_slots) {
            uint32_t h = place(slot);
            for (int had; (had = atomicCAS(&s_key[h], -1, slot)) != -1 && had != slot;) h = (h + 1) & (kTable - 1);
            atomicMax(&s_last[h], i);
            at = (int)h;
        }
        s_slot[i] = at;
    }
    __syncthreads();
    for (int r = r0 + rows + threadIdx.x; r < n_rows; r += 4 * kManyThreads) {
        int later[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) later[e] = r + e * kManyThreads < n_rows ? slots[r + e * kManyThreads] : -1;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if ((unsigned)later[e] >= (unsigned)n_slots) continue;
            uint32_t h = place(later[e]);
            for (int had; (had = s_key[h]) != -1; h = (h + 1) & (kTable - 1))
                if (had == later[e]) { s_last[h] = kManyRows; break; }       // none of this CTA's rows
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows; i += kManyThreads) {
        const int at = s_slot[i];
        s_slot[i] = at >= 0 && s_last[at] == i ? s_key[at] : -1;
    }
    __syncthreads();
    for (Walk at(threadIdx.x / 32, kManyThreads / 32, ((width + 127) / 128 + 2 * U - 1) / (2 * U)); at.row < 2 * rows; at.next()) {
        const int i = at.row >> 1, slot = s_slot[i];
        const bool keys = (at.row & 1) == 0;
        if (slot >= 0)
            store_segment<T, U>((keys ? k : v) + (r0 + i) * (keys ? ld_k : ld_v), keys ? wide_k : wide_v, slot, at.seg, keys ? k_codes : v_codes, keys ? k_scales : v_scales, width);
    }
}

template <typename T, int U>
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
    const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15, blocks = width / 32, quads = (blocks + 3) / 4;
    for (Walk at = warps_of_grid((quads + 2 * U - 1) / (2 * U)); at.row < n_rows; at.next()) {
        const int slot = slots ? slots[at.row] : at.row;
        if ((unsigned)slot >= (unsigned)n_slots) continue;
        const int quad0 = at.seg * 2 * U + half, col0 = quad0 * 128 + l * 8;
        const uint8_t *from = codes + (size_t)slot * (width / 2) + quad0 * 64 + l * 4, *s = scales + (size_t)slot * blocks + quad0 * 4 + (l >> 2);
        uint32_t w[U], c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            w[u] = c[u] = 0;
            if (col0 + u * 256 < width) { w[u] = *reinterpret_cast<const uint32_t *>(from + u * 128); c[u] = s[u * 8]; }
        }
        T *to = dst + at.row * ld + col0;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (col0 + u * 256 < width) {
                const uint4 x = mx4::decode8(w[u], c[u] > mx4::kCacheHi ? 255u : c[u]);
                if (wide) put(to + u * 256, x); else put_some(to + u * 256, x, 8);
            }
    }
}

// Pieces of a lane in a segment (2 U quads), one to four loads in flight: the longest segment that leaves at most a third of a row's lanes
// without work (40000 x 1280 fp32, 10 quads, to codes and back: 77 us at one piece, 63 at three; 40000 x 2688 bf16, 21 quads: 130 and 105 at
// four), an eighth where lanes shift their values together, which costs more than a load does (39518 x 3382, 27 quads: 233 us at three, 263 at
// four); else the one that leaves the fewest.
int pieces(int quads, bool wide)
{
    int best = 1, waste = 1 << 30;
    for (int u = 1; u <= 4; ++u) {
        const int w = (quads + 2 * u - 1) / (2 * u) * (2 * u) - quads;
        if (w * (wide ? 3 : 8) <= quads || w <= waste) { waste = w; best = u; }
    }
    return best;
}
int segments(int quads, bool wide) { const int u = pieces(quads, wide); return (quads + 2 * u - 1) / (2 * u); }
// the instance of a kernel template <T, U, ...> for so many pieces
#define SFS_BY_PIECES(kernel, u, ...) (u == 4 ? kernel<T, 4, ##__VA_ARGS__> : u == 3 ? kernel<T, 3, ##__VA_ARGS__> : u == 2 ? kernel<T, 2, ##__VA_ARGS__> : kernel<T, 1, ##__VA_ARGS__>)
bool wide_rows(const void *base, int64_t ld, size_t element) { return aligned_to(base, 16) && (ld * (int64_t)element) % 16 == 0; }
// CTAs for that many warps' segments: eight on an SM at most
unsigned grid_for(long long segs) { return (unsigned)std::max<long long>(1, std::min<long long>((segs + kWarps - 1) / kWarps, (long long)gemm_num_sms() * 8)); }

int short_lanes(int cols) { return cols <= 32 ? 4 : cols <= 64 ? 8 : cols <= 128 ? 16 : 32; }

template <typename T>
cudaError_t launch_quantize(const void *x, int64_t ldx, int rows, int cols, void *codes, int64_t ld_codes, void *scales, cudaStream_t stream)
{
    const int quads = (cols + 127) / 128;
    if (cols <= 256) {
        const int lanes = short_lanes(cols);
        const dim3 grid(grid_for(((long long)((rows + 127) / 128 * 128) * lanes / 32 + 3) / 4));
        auto kernel = lanes == 4 ? quantize_short_kernel<T, 4> : lanes == 8 ? quantize_short_kernel<T, 8> : lanes == 16 ? quantize_short_kernel<T, 16> : quantize_short_kernel<T, 32>;
        return launch_pdl(kernel, grid, dim3(kThreads), 0, stream, (const T *)x, (long long)ldx, rows, cols, (uint8_t *)codes, (long long)ld_codes, (uint8_t *)scales,
                          (int)wide_rows(x, ldx, sizeof(T)));
    }
    const bool wide = wide_rows(x, ldx, sizeof(T));
    const int u = pieces(quads, wide);
    const dim3 grid(grid_for((long long)((rows + 127) / 128 * 128) * segments(quads, wide)));
    return launch_pdl(wide ? SFS_BY_PIECES(quantize_kernel, u, true) : SFS_BY_PIECES(quantize_kernel, u, false), grid, dim3(kThreads), 0, stream, (const T *)x, (long long)ldx, rows, cols,
                      (uint8_t *)codes, (long long)ld_codes, (uint8_t *)scales, quads);
}
template <typename T>
cudaError_t launch_dequantize(const void *codes, int64_t ld_codes, const void *scales, int rows, int cols, void *x, int64_t ldx, cudaStream_t stream)
{
    const int quads = (cols + 127) / 128;
    if (cols <= 256) {
        const int lanes = short_lanes(cols);
        const dim3 grid(grid_for(((long long)rows * lanes / 32 + 3) / 4));
        auto kernel = lanes == 4 ? dequantize_short_kernel<T, 4> : lanes == 8 ? dequantize_short_kernel<T, 8> : lanes == 16 ? dequantize_short_kernel<T, 16> : dequantize_short_kernel<T, 32>;
        return launch_pdl(kernel, grid, dim3(kThreads), 0, stream, (const uint8_t *)codes, (long long)ld_codes, (const uint8_t *)scales, rows, cols, (T *)x, (long long)ldx,
                          (int)wide_rows(x, ldx, sizeof(T)));
    }
    const bool wide = wide_rows(x, ldx, sizeof(T));
    const int u = pieces(quads, wide);
    const dim3 grid(grid_for((long long)rows * segments(quads, wide)));
    return launch_pdl(wide ? SFS_BY_PIECES(dequantize_kernel, u, true) : SFS_BY_PIECES(dequantize_kernel, u, false), grid, dim3(kThreads), 0, stream, (const uint8_t *)codes,
                      (long long)ld_codes, (const uint8_t *)scales, rows, cols, (T *)x, (long long)ldx, quads);
}
// Rows up to which every CTA of a few compares all later slots with its own, and beyond which a table in shared memory holds more rows' (us,
// 8 heads of 128, scan / table; the calls' own 12 included): 2048 rows 18.5 / 19.1, 4096 23.5 / 21.4, 6144 31.3 / 23.2, 16384 98.8 / 33.1, 262144
// 17700 / 378; 32 heads: 2048 24.6 / 28.5, 4096 34.7 / 33.8, 6144 45.8 / 42.0.
constexpr int kFewSlots = 4096;
template <typename T>
cudaError_t launch_store(const sfs_cache4 &c, const void *k, int64_t ld_k, const void *v, int64_t ld_v, const int32_t *slots, int n_rows, cudaStream_t stream)
{
    const int width = c.n_kv_heads * c.head_dim, u = pieces((width + 127) / 128, true);
    const bool many = slots && n_rows > kFewSlots;
    // few rows: one or two for a CTA, so that they spread over the machine; many: two CTAs on an SM
    const int cta_rows = many ? std::min(kManyRows, (n_rows + 2 * gemm_num_sms() - 1) / (2 * gemm_num_sms())) : std::min(kStoreRows, std::max(1, n_rows / gemm_num_sms()));
    const dim3 grid((unsigned)((n_rows + cta_rows - 1) / cta_rows), many ? 1 : 2);
    return launch_pdl(many ? SFS_BY_PIECES(cache_store_many_kernel, u) : SFS_BY_PIECES(cache_store_kernel, u), grid, dim3(many ? kManyThreads : kThreads), 0, stream, (uint8_t *)c.k_codes,
                      (uint8_t *)c.k_scales, (uint8_t *)c.v_codes, (uint8_t *)c.v_scales, c.batch * c.capacity, width, (const T *)k, (long long)ld_k,
                      (const T *)v, (long long)ld_v, (int)wide_rows(k, ld_k, sizeof(T)), (int)wide_rows(v, ld_v, sizeof(T)), slots, n_rows, cta_rows);
}
template <typename T>
cudaError_t launch_load(const sfs_cache4 &c, const int32_t *slots, int n_rows, void *k, int64_t ld_k, void *v, int64_t ld_v, cudaStream_t stream)
{
    const int width = c.n_kv_heads * c.head_dim, quads = (width + 127) / 128;
    const int u = pieces(quads, true);
    const dim3 grid(grid_for((long long)n_rows * segments(quads, true)), 2);
    return launch_pdl(SFS_BY_PIECES(cache_load_kernel, u), grid, dim3(kThreads), 0, stream, (const uint8_t *)c.k_codes,
                      (const uint8_t *)c.k_scales, (const uint8_t *)c.v_codes, (const uint8_t *)c.v_scales, c.batch * c.capacity, width, (T *)k, (long long)ld_k,
                      (T *)v, (long long)ld_v, (int)wide_rows(k, ld_k, sizeof(T)), (int)wide_rows(v, ld_v, sizeof(T)), slots, n_rows);
}

}  // namespace

int32_t status_word_outside_captures(cudaStream_t stream, int32_t **word)
{
    if ((*word = device_status_word_if_any()) != nullptr) return SFS_OK;
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    SFS_CUDA(cudaStreamIsCapturing(stream, &capture));
    SFS_REQUIRE(capture == cudaStreamCaptureStatusNone, SFS_ERR_INVALID_ARG, "the first call on a device allocates its status word: make one before capturing a stream");
    SFS_REQUIRE((*word = device_status_word()) != nullptr, SFS_ERR_OOM, "cannot allocate the device status word");
    return SFS_OK;
}

int32_t cache4_check(const sfs_cache4 *c, const char *what)
{
    SFS_REQUIRE(c && c->k_codes && c->k_scales && c->v_codes && c->v_scales, SFS_ERR_INVALID_ARG, "%s: NULL cache", what);
    SFS_REQUIRE(aligned_to(c->k_codes, 16) && aligned_to(c->k_scales, 16) && aligned_to(c->v_codes, 16) && aligned_to(c->v_scales, 16),
                SFS_ERR_INVALID_ARG, "%s: codes and scales must be 16-byte aligned", what);
    SFS_REQUIRE(c->batch >= 1 && c->capacity >= 1 && c->n_kv_heads >= 1, SFS_ERR_INVALID_ARG, "%s: bad cache sizes", what);
    SFS_REQUIRE((int64_t)c->batch * c->capacity <= 0x7FFFFFFF, SFS_ERR_INVALID_ARG, "%s: more slots than an int32 names", what);
    SFS_REQUIRE(c->capacity <= (1 << 30), SFS_ERR_UNSUPPORTED, "%s: capacity above 2^30", what);
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
    SFS_REQUIRE((int64_t)rows * std::max(segments((cols + 127) / 128, false), segments((cols + 127) / 128, true)) < 0x7FFF0000, SFS_ERR_UNSUPPORTED, "mx4_quantize: matrix too large for one call");
    if (in_dtype == SFS_LOGITS_BF16) SFS_CUDA(launch_quantize<__nv_bfloat16>(d_x, ldx, rows, cols, d_codes, ld_codes, d_scales, (cudaStream_t)stream));
    else SFS_CUDA(launch_quantize<float>(d_x, ldx, rows, cols, d_codes, ld_codes, d_scales, (cudaStream_t)stream));
    return SFS_OK;
}

int32_t sfs_mx4_dequantize(const void *d_codes, int64_t ld_codes, const void *d_scales, int32_t rows, int32_t cols, void *d_x, int64_t ldx,
                           int32_t out_dtype, void *stream)
{
    const int32_t rc = check_matrix("mx4_dequantize", d_x, ldx, out_dtype, rows, cols, d_codes, ld_codes, d_scales);
    if (rc != SFS_OK) return rc;
    SFS_REQUIRE((int64_t)rows * std::max(segments((cols + 127) / 128, false), segments((cols + 127) / 128, true)) < 0x7FFF0000, SFS_ERR_UNSUPPORTED, "mx4_dequantize: matrix too large for one call");
    if (out_dtype == SFS_LOGITS_BF16) SFS_CUDA(launch_dequantize<__nv_bfloat16>(d_codes, ld_codes, d_scales, rows, cols, d_x, ldx, (cudaStream_t)stream));
    else SFS_CUDA(launch_dequantize<float>(d_codes, ld_codes, d_scales, rows, cols, d_x, ldx, (cudaStream_t)stream));
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
    SFS_REQUIRE(n_rows <= (1 << 30), SFS_ERR_UNSUPPORTED, "cache4_store: more than 2^30 rows");
    SFS_REQUIRE(aligned_to(d_slots, 4), SFS_ERR_INVALID_ARG, "cache4_store: misaligned slots");
    if ((rc = check_rows("cache4_store", cache, d_k, ld_k, in_dtype)) != SFS_OK || (rc = check_rows("cache4_store", cache, d_v, ld_v, in_dtype)) != SFS_OK) return rc;
    if (n_rows == 0) return SFS_OK;
    if (in_dtype == SFS_LOGITS_BF16) SFS_CUDA(launch_store<__nv_bfloat16>(*cache, d_k, ld_k, d_v, ld_v, d_slots, n_rows, (cudaStream_t)stream));
    else SFS_CUDA(launch_store<float>(*cache, d_k, ld_k, d_v, ld_v, d_slots, n_rows, (cudaStream_t)stream));
    return SFS_OK;
}

int32_t sfs_cache4_load(const sfs_cache4 *cache, const int32_t *d_slots, int32_t n_rows, void *d_k, int64_t ld_k, void *d_v, int64_t ld_v,
                        int32_t out_dtype, void *stream)
{
    int32_t rc = cache4_check(cache, "cache4_load");
    if (rc != SFS_OK) return rc;
    SFS_REQUIRE(out_dtype == SFS_LOGITS_BF16 || out_dtype == SFS_LOGITS_F32, SFS_ERR_INVALID_ARG, "cache4_load: type %d", out_dtype);
    SFS_REQUIRE(n_rows >= 0, SFS_ERR_INVALID_ARG, "cache4_load: n_rows %d", n_rows);
    SFS_REQUIRE(n_rows <= (1 << 30), SFS_ERR_UNSUPPORTED, "cache4_load: more than 2^30 rows");
    SFS_REQUIRE(aligned_to(d_slots, 4), SFS_ERR_INVALID_ARG, "cache4_load: misaligned slots");
    if (d_k && (rc = check_rows("cache4_load", cache, d_k, ld_k, out_dtype)) != SFS_OK) return rc;
    if (d_v && (rc = check_rows("cache4_load", cache, d_v, ld_v, out_dtype)) != SFS_OK) return rc;
    if (n_rows == 0 || (!d_k && !d_v)) return SFS_OK;
    if (out_dtype == SFS_LOGITS_BF16) SFS_CUDA(launch_load<__nv_bfloat16>(*cache, d_slots, n_rows, d_k, ld_k, d_v, ld_v, (cudaStream_t)stream));
    else SFS_CUDA(launch_load<float>(*cache, d_slots, n_rows, d_k, ld_k, d_v, ld_v, (cudaStream_t)stream));
    return SFS_OK;
}

}  // extern "C"

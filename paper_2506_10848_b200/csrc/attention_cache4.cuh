// Attention over a key / value cache of microscaled 4-bit numbers: arguments of its kernels.
#pragma once
#include "mx4.cuh"

namespace sfs {

struct Cache4Args {
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int batch, capacity, n_kv, group;                       // group: query heads per key head
    const __nv_bfloat16 *q; long long ld_q;
    __nv_bfloat16 *out; long long ld_out;
    int n_q;
    const int32_t *lengths, *positions;
    int left, right, sinks;
    float scale_log2;                                       // log2(e) / sqrt(head_dim)
    int32_t *err;
};

#ifdef __CUDACC__
__device__ __forceinline__ int cache4_length(const Cache4Args &a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.capacity) : a.capacity; }

// 16 bytes on their way to shared memory, of which the first `bytes` are read and the others 0
__device__ __forceinline__ void copy16(uint32_t smem, const void *global) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(global) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t smem, const void *global, int bytes) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(global), "r"(bytes) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// The keys that a query at position p sees: [0, first) and [lo, hi), first <= lo.
struct Seen { int first, lo, hi; };
__device__ __forceinline__ Seen cache4_seen(const Cache4Args &a, int length, long long p)
{
    Seen s;
    s.hi = a.right < 0 ? length : (int)min((long long)length, max(0ll, p + a.right + 1));
    s.lo = a.left < 0 ? 0 : (int)min((long long)s.hi, max(0ll, p - a.left));
    s.first = min(a.sinks, s.lo);
    return s;
}
#endif

// Rows are many: the tensor-memory kernel, and an estimate of its time.  `tokens`: how many a row sees at most.
int32_t attention_cache4_many(const Cache4Args &a, int64_t tokens, int head_dim, cudaStream_t stream);
double attention_cache4_many_us(const Cache4Args &a, int64_t tokens, int head_dim);
int32_t cache4_check(const sfs_cache4 *c, const char *what);

}  // namespace sfs

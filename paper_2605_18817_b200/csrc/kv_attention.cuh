// What the kernels on the paged key / value cache share: batch arguments and their checks, the workspace, how the
// attention's work is laid out over CTAs, and the joining of partial results.
#pragma once
#include "mrp_internal.cuh"

namespace mrp {

constexpr int kKvMaxSm = 160;              // SMs the workspace is sized for (a larger grid is clamped to it)

// Division by a fixed divisor 1 <= d < 2^31 of numbers below 2^31: n / d = (mulhi(n, mul) + n) >> shift.
struct FastDiv {
    uint32_t mul, shift;
    int32_t d;
};
inline FastDiv make_fastdiv(int32_t d)
{
    FastDiv f;
    uint32_t s = 0;
    while ((1ull << s) < (uint64_t)d) ++s;
    f.shift = s;
    f.mul = (uint32_t)(((1ull << 32) * ((1ull << s) - (uint64_t)d)) / (uint64_t)d + 1);
    f.d = d;
    return f;
}
__device__ __forceinline__ int fast_div(int n, const FastDiv &f)
{
    return (int)(((uint64_t)__umulhi((uint32_t)n, f.mul) + (uint32_t)n) >> f.shift);
}

// The batch and the pool as the kernels see them.
struct KvBatch {
    const int32_t *seq_start, *prefix_len, *page_table, *positions;
    int n_seqs, n_tokens, n_pages, max_pages;
    int cap;                   // positions a sequence can hold
    FastDiv page;              // page_size
    int64_t page_stride;       // elements
    int32_t *status, *user_status;
};

__device__ __forceinline__ void kv_bad_index(const KvBatch &b)
{
    atomicOr(b.status, MRP_DEV_BAD_INDEX);
    if (b.user_status) atomicOr(b.user_status, MRP_DEV_BAD_INDEX);
}

// Rows [start, start + n) of sequence s behind pre cached positions; false where they do not fit.
__device__ __forceinline__ bool kv_sequence(const KvBatch &b, int s, int &start, int &n, int &pre)
{
    start = __ldg(b.seq_start + s);
    const int end = __ldg(b.seq_start + s + 1);
    pre = __ldg(b.prefix_len + s);
    n = end - start;
    return start >= 0 && end >= start && end <= b.n_tokens && pre >= 0 && pre <= b.cap && n <= b.cap - pre;
}

// ---- workspace: arrival counters, then (max, sum) pairs and rows of partial results -----------------------------------
// Slot 2 c holds CTA c's part of a unit that an earlier CTA began, slot 2 c + 1 its part of one that a later CTA goes on
// with; a slot is `rows` rows of `width` floats and as many (max, sum) pairs.
constexpr int kKvCounterBytes = 4096;      // int32 per CTA that begins a shared unit; zero between calls
struct KvPartials {
    int32_t *counters;
    float2 *ml;
    float *o;
};

}  // namespace mrp

// Which sequence a row of the batch belongs to, and where its position lies in the pages.
#pragma once
#include "kv_attention.cuh"

namespace mrp {
namespace {

// Sequence of row t: the number of entries of seq_start[1..n_seqs] that are <= t, found by the warp 32 probes at a time
// (in 0..n_seqs whatever the list holds).
__device__ __forceinline__ int find_sequence(const int32_t *seq_start, int n_seqs, int t, int lane)
{
    int lo = 0, n = n_seqs;                // the answer lies in [lo, lo + n]
    while (n > 0) {
        const int step = (n + 31) / 32;
        const int at = lo + (lane + 1) * step - 1;
        const bool le = (lane + 1) * step - 1 < n && __ldg(seq_start + 1 + at) <= t;
        const int k = __popc(__ballot_sync(0xffffffffu, le));
        lo += k * step;
        n = min(step - 1, n - k * step);
    }
    return lo;
}

// The same where that list is not ascending (a sequence in it does not fit) or no sequence has the row: all of them; -1: none.
__device__ __noinline__ int scan_sequences(const KvBatch &b, int t, int lane)
{
    for (int s0 = 0; s0 < b.n_seqs; s0 += 32) {
        const int s = s0 + lane;
        int start, n, pre;
        const bool has = s < b.n_seqs && kv_sequence(b, s, start, n, pre) && t >= start && t - start < n;
        const uint32_t hit = __ballot_sync(0xffffffffu, has);
        if (hit) return s0 + __ffs(hit) - 1;
    }
    return -1;
}

// A sequence that does not fit is reported even if no row names it: once per launch, by one CTA.
__device__ __forceinline__ void report_sequences(const KvBatch &b, int tid, int threads)
{
    for (int s = tid; s < b.n_seqs; s += threads) {
        int start, n, pre;
        if (!kv_sequence(b, s, start, n, pre)) kv_bad_index(b);
    }
}

// The place of row t, found by a warp; false: no sequence that fits has the row.
struct TokenPlace {
    int pos;                   // position in the sequence
    int page, row;             // page entry (-1: outside the pool, reported) and row in it
};
__device__ __forceinline__ bool find_token(const KvBatch &b, int t, int lane, TokenPlace &at)
{
    int s = find_sequence(b.seq_start, b.n_seqs, t, lane);
    int start, n, pre;
    if (s >= b.n_seqs || !kv_sequence(b, s, start, n, pre) || t < start || t - start >= n) {
        s = scan_sequences(b, t, lane);
        if (s < 0) return false;
        kv_sequence(b, s, start, n, pre);
    }
    at.pos = pre + (t - start);
    const int pg = fast_div(at.pos, b.page);
    at.row = at.pos - pg * b.page.d;
    at.page = __ldg(b.page_table + (size_t)s * b.max_pages + pg);
    if ((unsigned)at.page >= (unsigned)b.n_pages) {
        if (lane == 0) kv_bad_index(b);
        at.page = -1;
    }
    return true;
}

}  // namespace
}  // namespace mrp

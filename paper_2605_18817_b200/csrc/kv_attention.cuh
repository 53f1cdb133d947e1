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

// Offsets on the line of tiles pass 32 bits only for enormous batches; their division is several times as long.
__device__ __forceinline__ long long div_line(long long a, long long b)
{
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// The batch and the pool as the kernels see them.
struct KvBatch {
    const int32_t *seq_start, *prefix_len, *page_table, *positions;
    int n_seqs, n_tokens, n_pages, max_pages;
    int cap;                   // positions a sequence can hold
    int beyond = 0;            // how far new tokens may lie behind them: 0, or any way where they need no place in the cache
    FastDiv page;              // page_size
    int64_t page_stride;       // elements
    int32_t *status, *user_status;
};

inline KvBatch kv_batch_of(const Ctx *c, const mrp_kv_batch &batch)
{
    KvBatch b;
    b.seq_start = batch.seq_start;
    b.prefix_len = batch.prefix_len;
    b.page_table = batch.page_table;
    b.positions = nullptr;
    b.n_seqs = batch.n_seqs;
    b.n_tokens = batch.n_tokens;
    b.n_pages = c->kv.n_pages;
    b.max_pages = c->kv.max_pages;
    b.cap = c->kv.max_pages * c->kv.page_size;
    b.page = make_fastdiv(c->kv.page_size);
    b.page_stride = c->kv.page_stride;
    b.status = (int32_t *)(c->ws + c->lay.status);
    b.user_status = batch.status;
    return b;
}

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
    pre = b.prefix_len ? __ldg(b.prefix_len + s) : 0;     // (no cache: nothing lies in front of the rows)
    n = end - start;
    return start >= 0 && end >= start && end <= b.n_tokens && pre >= 0 && pre <= b.cap && n <= b.cap + b.beyond - pre;
}

// ---- workspace: arrival counters, then (max, sum) pairs and rows of partial results -----------------------------------
// Slot 2 c holds CTA c's part of a unit that an earlier CTA began, slot 2 c + 1 its part of one that a later CTA goes on
// with; a slot is `rows` rows of `width` floats and as many (max, sum) pairs.
constexpr int kKvCounterBytes = 8192;      // int32 arrivals by the CTA that begins a shared unit (large tiles: per warp too); zero between
                                           // calls, also behind one whose wait gave up (settle_arrivals)
// Arrival behind a barrier of the threads that wrote: releases their stores, acquires those of the arrivals before.
__device__ __forceinline__ int arrive_acq_rel(int32_t *counter)
{
    int old;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
    return old;
}
struct KvPartials {
    int32_t *counters;
    float2 *ml;
    float *o;
};

// Where a kernel's keys and values lie: in pages of the context type, in rows beside the queries, in pages of 8 bits.
enum { kFromPages = 0, kFromRows = 1, kFromQ8 = 2 };

struct AttnParams {
    KvBatch b;
    const void *q, *k, *v;
    void *out;
    float *lse;
    int64_t q_stride, out_stride;
    int H, Hk, g, D;
    FastDiv gdiv;              // g
    int mask, window, sinks, plain_rows;
    int rows_above, rows_upto; // sequences with more than rows_above and at most rows_upto query rows a key head are this launch's
    int lead;                  // what a unit costs besides its tiles, in tiles: so much of the line lies ahead of each unit
    float scale_log2;          // > 0
    KvPartials part;
    int64_t k_stride, v_stride;                            // rows: elements from token to token
    int join;                  // rows: out and lse hold the result of a pass over other keys
    const uint8_t *k_scale, *v_scale;                      // 8 bits: scale bytes, of which there are scale_bytes
    int64_t scale_bytes;
};

// A row's sum over new keys (sum of p V with sum of p L at maximum m, base 2) beside the result of another pass (lse): out =
// a (sum of p V) + b (that pass's row).  b = 0 where that pass saw nothing: its row is not read then.
struct JoinWith {
    float a, b, lse;
};
__device__ __forceinline__ JoinWith join_with(float m, float L, float lse)
{
    const float l = L == 0.f ? -INFINITY : m + log2f(L), q = lse * 1.4426950408889634f;
    JoinWith j = {0.f, 0.f, -INFINITY};
    if (l == -INFINITY && q == -INFINITY) return j;
    const float top = fmaxf(l, q), x = exp2f(l - top), y = exp2f(q - top), s = x + y;      // (NaN goes through)
    j.a = L == 0.f ? 0.f : x / (s * L);
    j.b = y / s;
    j.lse = (top + log2f(s)) * 0.6931471805599453f;
    return j;
}

// whether position j lies in [lo, hi) or among the first `sinks` (below hi); no branches
__device__ __forceinline__ bool sees(int j, int hi, int lo, int sinks) { return (j < hi) & ((j >= lo) | (j < sinks)); }

// ---- the line of tiles ---------------------------------------------------------------------------------------------
// A row tile of a sequence: its rows, what they may see, its key tiles.  Tiles 0..first-1 hold the first positions that
// stay visible beside the window, the others start at key tile `base`.
template <int ROWS, int TILE> struct RowTile {
    int r0, rows;              // rows r0 .. r0 + rows - 1 of the sequence's n * g
    int lo, hi, s1;            // some row sees positions [lo, hi), [0, s1)
    int first, base, tiles;
};
template <int ROWS, int TILE>
__device__ __forceinline__ RowTile<ROWS, TILE> row_tile(const AttnParams &p, int n, int pre, int rt)
{
    RowTile<ROWS, TILE> t;
    t.r0 = rt * ROWS;
    t.rows = min(ROWS, n * p.g - t.r0);
    const int i0 = fast_div(t.r0, p.gdiv), i1 = fast_div(t.r0 + t.rows - 1, p.gdiv);
    t.hi = p.mask == MRP_ATTN_CAUSAL ? pre + i1 + 1 : p.mask == MRP_ATTN_BLOCK ? pre + n : pre;
    t.lo = p.window > 0 ? max(0, pre + i0 + 1 - p.window) : 0;
    t.s1 = p.window > 0 ? min(min(p.sinks, t.lo), t.hi) : 0;
    t.base = t.lo / TILE;
    const int end = t.hi > t.lo ? (t.hi + TILE - 1) / TILE : t.base;
    t.first = (t.s1 + TILE - 1) / TILE;
    if (t.first >= t.base) {               // they meet: one run from position 0
        t.tiles = max(end > t.base ? end : 0, t.first);
        t.first = 0;
        t.base = 0;
    } else {
        t.tiles = t.first + (end - t.base);
    }
    t.tiles = max(t.tiles, 1);             // rows that see nothing are still written
    return t;
}
template <int ROWS, int TILE>
__device__ __forceinline__ int key_tile(const RowTile<ROWS, TILE> &t, int i) { return i < t.first ? i : t.base + i - t.first; }

__device__ __forceinline__ bool takes(const AttnParams &p, int n)
{
    const long long rows = (long long)n * p.g;
    return rows > p.rows_above && rows <= p.rows_upto;
}

template <int ROWS, int TILE>
__device__ __forceinline__ long long sequence_tiles(const AttnParams &p, int s, bool report)
{
    int start, n, pre;
    if (!kv_sequence(p.b, s, start, n, pre)) {
        if (report) kv_bad_index(p.b);
        return 0;
    }
    if (!takes(p, n)) return 0;
    const int nrt = (n * p.g + ROWS - 1) / ROWS;
    long long sum = 0;
    for (int rt = 0; rt < nrt; ++rt) sum += row_tile<ROWS, TILE>(p, n, pre, rt).tiles + p.lead;
    return sum * p.Hk;
}

// A place on the line: place `i` of unit (sequence s, row tile rt, key head h), tile i - lead of it from i = lead on; `at` its
// offset on the line, `unit` the offset of the unit's first place.
template <int ROWS, int TILE> struct Cursor {
    int s, rt, h, i;
    int start, n, pre;
    RowTile<ROWS, TILE> t;
    long long at, unit;
};
template <int ROWS, int TILE>
__device__ __forceinline__ bool open_sequence(const AttnParams &p, Cursor<ROWS, TILE> &c)
{
    for (; c.s < p.b.n_seqs; ++c.s)
        if (kv_sequence(p.b, c.s, c.start, c.n, c.pre) && takes(p, c.n)) {
            c.rt = 0; c.h = 0; c.i = 0;
            c.t = row_tile<ROWS, TILE>(p, c.n, c.pre, 0);
            return true;
        }
    return false;
}
template <int ROWS, int TILE>
__device__ __forceinline__ void advance(const AttnParams &p, Cursor<ROWS, TILE> &c)
{
    ++c.at;
    if (++c.i < c.t.tiles + p.lead) return;
    c.i = 0;
    c.unit = c.at;
    if (++c.h < p.Hk) return;
    c.h = 0;
    if (++c.rt < (c.n * p.g + ROWS - 1) / ROWS) {
        c.t = row_tile<ROWS, TILE>(p, c.n, c.pre, c.rt);
        return;
    }
    ++c.s;
    open_sequence(p, c);
}

// The unit at `c`, as far as it lies in a piece that ends at piece_end: places, of which tiles begin .. begin + count - 1.
struct UnitPart {
    int places, begin, count;
};
template <int ROWS, int TILE>
__device__ __forceinline__ UnitPart unit_part(const AttnParams &p, const Cursor<ROWS, TILE> &c, long long piece_end)
{
    UnitPart u;
    u.places = (int)min((long long)(c.t.tiles + p.lead - c.i), piece_end - c.at);
    u.begin = max(0, c.i - p.lead);
    u.count = max(0, c.i + u.places - p.lead) - u.begin;
    return u;
}
// On to the next unit, behind the `places` of this one.
template <int ROWS, int TILE>
__device__ __forceinline__ void leave_unit(const AttnParams &p, Cursor<ROWS, TILE> &c, int places, long long piece_end)
{
    c.at += places;
    if (c.at < piece_end) {
        c.i = c.t.tiles + p.lead - 1;
        --c.at;
        advance(p, c);
    }
}
// The CTAs that hold tiles of the unit at `c`, by the length `per` of their pieces.
template <int ROWS, int TILE>
__device__ __forceinline__ void unit_pieces(const AttnParams &p, const Cursor<ROWS, TILE> &c, long long per, int &c0, int &c1)
{
    c0 = (int)div_line(c.unit + p.lead, per);
    c1 = (int)div_line(c.unit + p.lead + c.t.tiles - 1, per);
}

// What a CTA that leaves early (a wait gave up) still owes: an arrival at each cut unit it holds tiles of, from the unit at `c`
// to the end of its piece, so that the counters come back to zero and the next call's pieces are not joined early.
// `arrive(c, c0, c1)` counts one of the c1 - c0 + 1 arrivals and clears the counter at the last; nothing is joined.
template <int ROWS, int TILE, typename F>
__device__ __forceinline__ void settle_arrivals(const AttnParams &p, Cursor<ROWS, TILE> &c, long long per, long long piece_end, F arrive)
{
    while (c.at < piece_end) {
        const UnitPart u = unit_part(p, c, piece_end);
        if (u.count > 0 && u.count < c.t.tiles) {
            int c0, c1;
            unit_pieces(p, c, per, c0, c1);
            arrive(c, c0, c1);
        }
        leave_unit(p, c, u.places, piece_end);
    }
}

// Sets `c` to the start of this CTA's piece and returns its length; `per` is the length of a full piece.
template <int ROWS, int TILE, int THREADS>
__device__ __forceinline__ long long find_piece(const AttnParams &p, Cursor<ROWS, TILE> &c, long long &per, long long *sh)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int WARPS = THREADS / 32;
    long long *sh_warp = sh, *sh_found = sh + WARPS;      // [WARPS], [2]
    long long total = 0, mine = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += THREADS) {
        const int s = s0 + tid;
        mine = s < p.b.n_seqs ? sequence_tiles<ROWS, TILE>(p, s, blockIdx.x == 0) : 0;
        long long x = mine;
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
        __syncthreads();
        if (lane == 0) sh_warp[warp] = x;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) total += sh_warp[w];
    }
    per = div_line(total + gridDim.x - 1, gridDim.x);
    const long long begin = per * blockIdx.x, end = min(total, begin + per);
    if (begin >= end) return 0;
    long long done = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += THREADS) {
        const int s = s0 + tid;
        if (p.b.n_seqs > THREADS) mine = s < p.b.n_seqs ? sequence_tiles<ROWS, TILE>(p, s, false) : 0;
        long long x = mine;                // inclusive sum over the lanes
#pragma unroll
        for (int w = 1; w < 32; w <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, w);
            if (lane >= w) x += y;
        }
        __syncthreads();
        if (lane == 31) sh_warp[warp] = x;
        __syncthreads();
        long long before = done + x - mine;
        for (int w = 0; w < warp; ++w) before += sh_warp[w];
        for (int w = 0; w < WARPS; ++w) done += sh_warp[w];
        if (mine > 0 && before <= begin && begin < before + mine) {
            sh_found[0] = s;
            sh_found[1] = before;
        }
        __syncthreads();
        if (done > begin) break;
    }
    c.s = (int)sh_found[0];
    c.at = sh_found[1];
    open_sequence(p, c);
    while (c.at + (long long)(c.t.tiles + p.lead) * p.Hk <= begin) {
        c.at += (long long)(c.t.tiles + p.lead) * p.Hk;
        c.t = row_tile<ROWS, TILE>(p, c.n, c.pre, ++c.rt);
    }
    const int in = (int)(begin - c.at);
    c.h = in / (c.t.tiles + p.lead);
    c.i = in - c.h * (c.t.tiles + p.lead);
    c.at = begin;
    c.unit = begin - c.i;
    return end - begin;
}

// The same for a warp on its own, for up to 128 sequences: no barrier, and the sequence's numbers come from the lane that
// has them.
template <int ROWS, int TILE>
__device__ __forceinline__ long long find_piece_warp(const AttnParams &p, Cursor<ROWS, TILE> &c, long long &per, bool report)
{
    const int lane = threadIdx.x & 31;
    int start[4], n[4], pre[4];
    long long tiles[4], total = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        start[i] = n[i] = pre[i] = 0;
        tiles[i] = 0;
        if (32 * i < p.b.n_seqs) {
            const int s = lane + 32 * i;
            if (s < p.b.n_seqs) {
                if (kv_sequence(p.b, s, start[i], n[i], pre[i])) {
                    const int nrt = takes(p, n[i]) ? (n[i] * p.g + ROWS - 1) / ROWS : 0;
                    for (int rt = 0; rt < nrt; ++rt) tiles[i] += row_tile<ROWS, TILE>(p, n[i], pre[i], rt).tiles + p.lead;
                    tiles[i] *= p.Hk;
                } else if (report) {
                    kv_bad_index(p.b);
                }
            }
            total += tiles[i];
        }
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) total += __shfl_xor_sync(0xffffffffu, total, w);
    per = div_line(total + gridDim.x - 1, gridDim.x);
    const long long begin = per * blockIdx.x, end = min(total, begin + per);
    if (begin >= end) return 0;
    long long done = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (32 * i < p.b.n_seqs && done <= begin) {
            long long x = tiles[i];
#pragma unroll
            for (int w = 1; w < 32; w <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, w);
                if (lane >= w) x += y;
            }
            const long long before = done + x - tiles[i];
            const uint32_t hit = __ballot_sync(0xffffffffu, tiles[i] > 0 && before <= begin && begin < before + tiles[i]);
            if (hit) {
                const int from = __ffs(hit) - 1;
                c.s = 32 * i + from;
                c.at = __shfl_sync(0xffffffffu, before, from);
                c.start = __shfl_sync(0xffffffffu, start[i], from);
                c.n = __shfl_sync(0xffffffffu, n[i], from);
                c.pre = __shfl_sync(0xffffffffu, pre[i], from);
            }
            done += __shfl_sync(0xffffffffu, x, 31);
        }
    c.rt = 0;
    c.t = row_tile<ROWS, TILE>(p, c.n, c.pre, 0);
    while (c.at + (long long)(c.t.tiles + p.lead) * p.Hk <= begin) {
        c.at += (long long)(c.t.tiles + p.lead) * p.Hk;
        c.t = row_tile<ROWS, TILE>(p, c.n, c.pre, ++c.rt);
    }
    const int in = (int)(begin - c.at);
    c.h = in / (c.t.tiles + p.lead);
    c.i = in - c.h * (c.t.tiles + p.lead);
    c.at = begin;
    c.unit = begin - c.i;
    return end - begin;
}

// The kernel on large tiles (kv_attention_tc.cu): the geometries it takes, its workspace, its launch.
bool kv_tc_takes(const mrp_config &cfg, const mrp_kv_config &kv);
bool kv_tc_any(const mrp_config &cfg, const mrp_kv_config &kv);
size_t kv_tc_workspace_bytes();
cudaError_t kv_tc_attach(Ctx *c);
cudaError_t launch_paged_attention_tc(Ctx *c, AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st);
bool kv_tc_takes_q8(const mrp_config &cfg, const mrp_kv_config &kv);
cudaError_t launch_paged_attention_q8_tc(Ctx *c, AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st);
cudaError_t kv_few_q8_prepare();
cudaError_t launch_few_q8(Ctx *c, AttnParams &p, int box_rows, bool eight, cudaStream_t st);    // (kv_attention_q8.cu)
bool kv_tc_takes_rows(const mrp_config &cfg, const mrp_kv_config &kv, const mrp_packed_kv &rows);
cudaError_t kv_short_prepare();
cudaError_t launch_packed_attention_short(Ctx *c, const AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st);      // (kv_attention_short.cu)
cudaError_t launch_packed_attention_tc(Ctx *c, AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st);

}  // namespace mrp

// Attention over pages of 8 bits, up to 16 query rows a sequence and key head: kv_attention_few_kernel (kv_attention_tc.cu, whose
// mathematics and units' ends these are) with half the bytes to read, which leaves half the time for everything else.
//
//   S^T = K Q^T on the codes as they lie: K's tile is the A operand in e4m3 (kind::f8f6f4), and a query row is two e4m3 rows of B,
//   q = 2^E (hi + lo / 16): eight significant bits, which is all of a bf16 (elements below 2^-13 of their row's largest: to 2^-21 of
//   that).  The thread that has a key takes its score times 2^E of the row times the key's scale.
//   O^T += V^T P^T in bf16: warps turn the codes of V times their scales into bf16 (exact) in two stages of their own.  In 8 bits
//   P would need three parts or more, and lose the tail of a long cache, whose many small probabilities lie below what e4m3 holds.
//   Turning K too would move 3 bytes more through shared memory for each of its codes, which then bounds the kernel instead of
//   memory: TMA, warps and MMAs move 88 of 128 bytes a cycle at the memory's rate as it is.
//
//   warp 0   K by TMA, and its scales      warp 1   S MMAs      warp 2   PV MMAs      warp 3   V and its scales
//   warps 4-7, 8-11   softmax, a thread per key and eight rows: two warpgroups that take tiles in turn (8 rows; maxima, sums and
//            accumulators of their own, joined at the unit's end) or the same tiles' rows by halves (16 rows: 32 blocks of 4 take 67 us
//            either way, but a thread's 16 rows would need 100 registers and leave room for four turning warps instead of eight)
//   warps 12-15   queries, a unit ahead, and units' ends          from warp 16 on   V's codes -> bf16 (two groups of four warps, a stage each)
// Instructions bound it next to memory, so each role's loop is short: the roles of an SM quarter share its instruction cache and
// its issue slots.  (One warp for both kinds of MMAs, scales looked up by the warps that use them, turning unrolled: 64 ragged
// single tokens 266 us; the turning rolled and 8 rows instead of 16: 159.)
// Measured, in a graph: 64 ragged single tokens of up to 9000 positions, 32 / 8 heads of 128: 130 us for 623 MB, 4.8 TB/s (issue
// slots 48 % busy, DRAM 58 %); 32 blocks of 4 behind 200 to 6000 positions 67 us; one token behind 2500, 16 / 8 heads 14 us, which is
// the chain of start, cut of the line, page entries, a tile and the join of 16 pieces, none of it wide.
// Clock reads at the barriers: with 8 rows the fetching warps are the busiest (they wait for room 22 % of the time, the S warp 45 % for K,
// the softmax 46 %, the turning warps 54 %), with 16 rows the softmax (waits 17 %; the turning warps 50 % for a stage).
#include "kv_tile.cuh"

namespace mrp {
namespace {

// A head is HB blocks of 128 features; a unit has up to ROWS query rows, 8 or 16.
template <int HB, int ROWS> struct FewQ8Geo {
    static constexpr int NR = ROWS;
    static constexpr int kCols = 2 * NR;                   // columns of S (hi, lo of Q), of P (hi, lo) and of an accumulator
    // of 128 keys, 128 codes: as much in flight as there is room for (three and four: 64 ragged 139 us).  Raw stages are even in number:
    // a stage belongs to one group of the turning warps then, which waits for every one of its phases.  With an odd number a group
    // could come to a stage whose phase before, the other group's, is still open, and take it for its own.
    static constexpr int kKStages = HB + NR / 8 == 3 ? 4 : 5, kRawStages = HB + NR / 8 == 4 ? 2 : 4;
    static_assert(kRawStages % 2 == 0, "a group of turning warps a raw stage");
    static constexpr int kRawAt = kKStages * 16384;
    static constexpr int kVAt = kRawAt + kRawStages * 16384;               // two stages of bf16 V
    static constexpr int kPRow = kCols * 2, kP = 128 * kPRow;              // P of a warpgroup: 128 keys, rows of 32 or 64 swizzled bytes
    static constexpr int kQ = HB * kCols * 128;            // queries of a unit, two of them
    static constexpr int kPAt = kVAt + 2 * 32768, kQAt = kPAt + 2 * kP, kBars = kQAt + 2 * kQ;
    static constexpr int kSmem = kBars + 1024 + 1024;      // + alignment of the base
    static constexpr int kTmem = NR == 16 ? 512 : 256;     // of which 8 kCols (S) + 4 HB kCols are used
    static constexpr int kTurners = 8;                     // warps
    static constexpr bool kSplit = NR == 16;               // both warpgroups take every tile, eight rows each
    static constexpr int kThreads = 512 + 32 * kTurners;
    static constexpr int kWide = HB * 128;                 // features of a row of partial results
};

// The unit's query rows as two e4m3 parts each (row r: hi, row NR + r: lo), K-major blocks of 128 features, and what their scores
// are multiplied by: 2^E scale log2(e), NaN for a row that is not finite.  128 threads, 128 / NR a row.
template <int HB, int NR>
__device__ __forceinline__ void load_query_parts(const AttnParams &p, int start, int h, int r0, int rows, uint32_t sq, float *factor, int tid)
{
    constexpr int kParts = 128 / NR, kChunks = 16 * HB / kParts;           // threads a row; runs of 8 features a thread
    const int r = tid / kParts, part = tid % kParts;
    const int rr = r0 + min(r, rows - 1), tok = fast_div(rr, p.gdiv), hg = rr - tok * p.g;
    const uint4 *src = reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(p.q) + (int64_t)(start + tok) * p.q_stride + (int64_t)(h * p.g + hg) * p.D);
    const int have = r < rows ? p.D / 8 : 0;
    uint4 x[kChunks];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = part + kParts * i;
        x[i] = c < have ? __ldg(src + c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int y = 0; y < 4; ++y) top = max(top, max((w[y] << 16) & 0x7FFFFFFFu, w[y] & 0x7FFF0000u));
    }
#pragma unroll
    for (int w = 1; w < kParts; w <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
    const uint32_t s = q8_scale(top);
    const bool fine = s != kQ8NaN;
    const float inv = q8_inverse(fine ? s : 127u);
    if (part == 0) factor[r] = q8_factor(s) * p.scale_log2;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = part + kParts * i;
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            float f[4] = {__uint_as_float(w[2 * y] << 16), __uint_as_float(w[2 * y] & 0xFFFF0000u), __uint_as_float(w[2 * y + 1] << 16),
                          __uint_as_float(w[2 * y + 1] & 0xFFFF0000u)};
#pragma unroll
            for (int z = 0; z < 4; ++z) f[z] = fine ? f[z] * inv : 0.f;
            hi[y] = q8_codes(f[0], f[1], f[2], f[3]);
            const float2 a = q8_values(hi[y] & 0xFFFFu, 1.f), b = q8_values(hi[y] >> 16, 1.f);
            lo[y] = q8_codes((f[0] - a.x) * 16.f, (f[1] - a.y) * 16.f, (f[2] - b.x) * 16.f, (f[3] - b.y) * 16.f);
        }
        // features 8 c .. of a block of 128: half of a 16-byte chunk, swizzled by the row (rows r and NR + r alike)
        const int cb = c & 15;
        const uint32_t at = sq + (c >> 4) * (2 * NR * 128) + r * 128 + ((((cb >> 1) ^ (r & 7)) << 4) | ((cb & 1) << 3));
        asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(hi[0]), "r"(hi[1]) : "memory");
        asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at + NR * 128), "r"(lo[0]), "r"(lo[1]) : "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// 8 columns each of the warp's 32 lanes, from two places
__device__ __forceinline__ void tmem_ld8_two(uint32_t a, uint32_t b, float *v, float *w)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v), *s = reinterpret_cast<uint32_t *>(w);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(a) : "memory");
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(s[0]), "=r"(s[1]), "=r"(s[2]), "=r"(s[3]), "=r"(s[4]), "=r"(s[5]), "=r"(s[6]), "=r"(s[7]) : "r"(b) : "memory");
    tmem_wait_ld();
    asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                      "+f"(w[0]), "+f"(w[1]), "+f"(w[2]), "+f"(w[3]), "+f"(w[4]), "+f"(w[5]), "+f"(w[6]), "+f"(w[7]) :: "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t a, const float *v)
{
    const uint32_t *r = reinterpret_cast<const uint32_t *>(v);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// P^T as the B operand: rows (keys) of 32 or 64 bytes, MN-major, swizzled over as many
template <int ROW> __device__ __forceinline__ uint64_t p_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(8 * ROW >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)(ROW == 32 ? 6 : 4) << 61;
}

// 4 bytes to shared memory, which arrive at the barrier when they are there (zeros where !on)
__device__ __forceinline__ void copy_word(uint32_t dst, const void *src, bool on, uint32_t bar)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// The scale bytes of a lane's four keys of V at a boundary of what is seen: see the scales' warp.
template <typename Tile>
__device__ __noinline__ uint32_t mend_scales(const Tile &t, const Seen &a, int j0, uint32_t w, Suspects &sus, int lane, bool tell)
{
    uint32_t keep = 0, bad = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int j = j0 + lane * 4 + e;
        const bool seen = j < t.hi && (j >= t.lo || j < t.s1), nan = ((w >> (8 * e)) & 255u) == kQ8NaN;
        const bool some = seen && nan && a.differ && !(j >= a.all_lo && j < a.all_hi);
        bad |= (uint32_t)some << e;
        keep |= seen && !some ? 255u << (8 * e) : 0u;
    }
    if (tell && __any_sync(0xffffffffu, bad != 0)) {
        const int slot = sus.n;
        __syncwarp();
        if (lane == 0) sus.n = slot + 1;
        if (slot < kMaxSuspects) {
            if (lane == 0) sus.base[slot] = j0;
            uint32_t word = bad << (4 * (lane & 7));       // 32 keys, of eight lanes
#pragma unroll
            for (int x = 1; x < 8; x <<= 1) word |= __shfl_xor_sync(0xffffffffu, word, x);
            if ((lane & 7) == 0) sus.keys[slot][lane >> 3] = word;
        }
        __syncwarp();
    }
    return w & keep;
}

template <int HB, int NR>
__global__ void __launch_bounds__(FewQ8Geo<HB, NR>::kThreads, 1)
kv_attention_few_q8_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap kmap,
                           const __grid_constant__ CUtensorMap vmap, const PageBoxes bx)
{
    typedef FewQ8Geo<HB, NR> G;
    typedef RowTile<NR, kTcTile> Tile;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Cursor<NR, kTcTile> sh_cur;                 // where this CTA's piece of the line begins, its length, a full piece's
    __shared__ long long sh_len, sh_per;
    __shared__ Suspects suspects[2];
    __shared__ uint32_t sh_ks[8][32], sh_vs[G::kRawStages][32];            // scale bytes of the keys of a tile's K (by S buffer), of a raw stage
    __shared__ int sh_hi[2][NR], sh_lo[2][NR];             // what a row sees: [lo, hi) and the first positions
    constexpr int kR = 8;                                  // rows of a warpgroup
    constexpr int kStep = G::kSplit ? 1 : 2;               // from one of its tiles to the next
    __shared__ __align__(16) float sh_ms[2][2][kR], sh_c[2][kR], sh_rf[2][NR];     // maximum in use (unit, warpgroup), factor to it; rows' factors
    __shared__ float sh_wm[2][4][kR], sh_wl[2][2][4][kR];  // row maxima and (of a unit) sums of the warps
    __shared__ float sh_f[2][NR];                          // the unit's end: factors of the accumulators,
    __shared__ int64_t sh_out[NR];                         //   where the rows go
    __shared__ int sh_last;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bars = base + G::kBars;
    auto k_at = [&](int s) { return base + s * 16384; };           // codes of K: operand stages
    auto r_at = [&](int s) { return base + G::kRawAt + s * 16384; };       // codes of V, raw
    auto v_at = [&](int s) { return base + G::kVAt + s * 32768; };         // V in bf16
    auto k_full = [&](int s) { return bars + 8 * s; };
    auto k_empty = [&](int s) { return bars + 8 * (6 + s); };
    auto raw_full = [&](int s) { return bars + 8 * (12 + s); };    // the codes, and their scales
    auto raw_empty = [&](int s) { return bars + 8 * (16 + s); };
    auto v_full = [&](int s) { return bars + 8 * (20 + s); };
    auto v_empty = [&](int s) { return bars + 8 * (22 + s); };
    auto s_full = [&](int b) { return bars + 8 * (40 + b); };      // the scores of a tile, and the keys' scales
    auto s_free = [&](int b) { return bars + 8 * (48 + b); };
    auto p_ready = [&](int x) { return bars + 8 * (28 + x); };
    auto pv_done = [&](int x) { return bars + 8 * (30 + x); };
    auto q_ready = [&](int x) { return bars + 8 * (32 + x); };
    auto unit_end = [&](int x) { return bars + 8 * (34 + x); };    // the unit is written: everything of it may be reused
    auto acc_full = [&](int x) { return bars + 8 * (36 + x); };    // the unit's sums, maxima and accumulators are there
    unsigned char *gbars = smem_raw + (base - smem_u32(smem_raw)) + G::kBars;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(gbars + 8 * 56);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    const WaitStatus ws = {p.b.status, p.b.user_status};

    if (tid == 0) {
        for (int s = 0; s < G::kKStages; ++s) {
            mbar_init(k_full(s), 1);
            mbar_init(k_empty(s), 1);
        }
        for (int s = 0; s < G::kRawStages; ++s) {
            mbar_init(raw_full(s), 33);
            mbar_init(raw_empty(s), 4);
        }
        for (int b = 0; b < 8; ++b) {
            mbar_init(s_full(b), 33);
            mbar_init(s_free(b), G::kSplit ? 8 : 4);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(v_full(x), 4);
            mbar_init(v_empty(x), 1);
            mbar_init(p_ready(x), G::kSplit ? 8 : 4);
            mbar_init(pv_done(x), 1);
            mbar_init(q_ready(x), 128);
            mbar_init(unit_end(x), 4);
            mbar_init(acc_full(x), 9);
        }
        *abort_flag = 0;
        prefetch_tmap(&kmap);
        prefetch_tmap(&vmap);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"((uint32_t)G::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 2) {
        pdl_wait();
        Cursor<NR, kTcTile> c;
        long long full = 1;
        c.at = 0;
        const long long len = cut_line<NR>(p, c, full, blockIdx.x == 0);
        if (lane == 0) {
            sh_cur = c;
            sh_len = len;
            sh_per = full;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;    // eight buffers of S, then accumulators of two units (8 rows: of each warpgroup)
    auto s_at = [&](int b) { return tmem + b * G::kCols; };        // (columns: the upper parts of the rows, the lower ones)
    auto o_at = [&](int u, int x) { return tmem + 8 * G::kCols + (2 * u + x) * HB * G::kCols; };    // (HB accumulators of 128 features)
    pdl_wait();
    pdl_trigger();

    Cursor<NR, kTcTile> cur = sh_cur;
    const long long per = sh_per, piece_end = sh_len > 0 ? cur.at + sh_len : 0;
    if (sh_len == 0) cur.at = 0;
    bool ok = true;
    auto to_tiles = [&](Cursor<NR, kTcTile> &c) {          // on to a unit that this piece has tiles of
        while (c.at < piece_end) {
            const UnitPart part = unit_part(p, c, piece_end);
            if (part.count > 0) break;
            next_unit(p, c, part.places, piece_end);
        }
    };
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, ws)); };   // a warp's

    if (warp == 0 || warp == 3) {
        // ================================ K (warp 0), V (warp 3): tiles and their scales ================================
        // A lane has a box of one of the next tiles (32 lanes: 2 to 32 tiles), so that what it takes to find a page, and its latency,
        // comes once a box and not once a lane and tile (64 ragged single tokens 137 us so).  Scales go a word of four keys a lane,
        // copied asynchronously.  V rows that must not reach the product get scale byte 0 here (their probabilities are 0, and the
        // codes times 2^-127 are finite): those no row sees, and rows of NaN that some see and others do not (remembered: the
        // output of those that do is NaN).
        const bool v = warp == 3;
        const uint8_t *scale = v ? p.v_scale : p.k_scale;
        const int pitch = v ? min(p.D, 128) : 128, stages = v ? G::kRawStages : G::kKStages;
        const uint32_t at = v ? r_at(0) : k_at(0), full = v ? raw_full(0) : k_full(0), empty = v ? raw_empty(0) : k_empty(0);
        const int log_rows = 31 - __clz(bx.rows), log_boxes = 7 - log_rows, boxes = 1 << log_boxes, tiles = 32 >> log_boxes;
        const int my_tile = lane >> log_boxes, my_box = lane & (boxes - 1);
        uint32_t unit = 0, k = 0, phase = 0;
        int stage = 0;
        struct Box {
            int entry, row;                                // entry -1: not needed
        };
        auto find = [&](const Cursor<NR, kTcTile> &c, const UnitPart &part, int n) {       // the lane's box of tiles n ..
            const int j = key_tile(c.t, part.begin + n + my_tile) * kTcTile + (my_box << log_rows);
            Box b = {-1, 0};
            if (n + my_tile < part.count && ((j < c.t.hi && j + bx.rows > c.t.lo) || j < c.t.s1)) {
                const int pg = fast_div(j, p.b.page);
                b.row = j - pg * p.b.page.d;
                b.entry = __ldg(p.b.page_table + (size_t)c.s * p.b.max_pages + pg);
                if (b.entry < 0) b.entry = p.b.n_pages;
            }
            return b;
        };
        to_tiles(cur);
        Box next = {-1, 0};
        if (cur.at < piece_end) next = find(cur, unit_part(p, cur, piece_end), 0);
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            const Tile t = cur.t;
            const Seen all = seen_by_all(p, t, cur.pre);
            const int u = unit & 1, h = cur.h;
            const int lo = all.differ ? max(t.lo, all.all_lo) : t.lo, hi = all.differ ? min(t.hi, all.all_hi) : t.hi;     // tiles in here: all is seen by all
            if (v) {
                if (unit >= 2) wait(unit_end(u), ((unit >> 1) - 1u) & 1u);         // (the suspects of the unit before the last)
                if (lane == 0) suspects[u].n = 0;
                __syncwarp();
            }
#pragma unroll 1
            for (int n0 = 0; n0 < count && ok; n0 += tiles) {
                const Box box = next;
                const bool need = box.entry >= 0, fine = need && box.entry < p.b.n_pages;
                if (need && !fine) kv_bad_index(p.b);
                const int page = fine ? box.entry : p.b.n_pages;                   // (a page that is not one: outside the map, zeros arrive)
                const int64_t scales = fine ? ((int64_t)box.entry * p.Hk + h) * p.b.page.d + box.row : -1;
                const uint32_t needed = __ballot_sync(0xffffffffu, need);
                if (n0 + tiles < count) next = find(cur, part, n0 + tiles);
#pragma unroll 1
                for (int i = 0; i < min(tiles, count - n0) && ok; ++i, ++k) {
                    const uint32_t here = (needed >> (i << log_boxes)) & (uint32_t)((1ull << boxes) - 1);
                    // the word of the lane's keys 4 l .. 4 l + 3 (no page, not needed: zeros, as its codes or whatever they are)
                    const int64_t from = __shfl_sync(0xffffffffu, scales, (i << log_boxes) | ((lane * 4) >> log_rows));
                    const uint8_t *word = scale + (from < 0 ? 0 : from + ((lane * 4) & (bx.rows - 1)));
                    if (!v) {
                        const uint32_t b = k & 7u;
                        wait(s_free(b), ((k >> 3) & 1u) ^ 1u);
                        copy_word(smem_u32(&sh_ks[b][lane]), word, from >= 0, s_full(b));
                    }
#pragma unroll
                    for (int y = 0; y < HB; ++y) {
                        const uint32_t bar = full + 8 * stage;
                        wait(empty + 8 * stage, phase ^ 1u);
                        if (!ok) break;
                        if (lane == 0) mbar_expect_tx(bar, __popc(here) * (uint32_t)(bx.rows * pitch));
                        __syncwarp();
                        if (my_tile == i && need)
                            tma_load_page(at + stage * 16384 + (my_box << log_rows) * pitch, v ? &vmap : &kmap, 128 * y, box.row, h, page, bar);
                        if (v) {
                            const int j0 = key_tile(t, begin + n0 + i) * kTcTile;
                            if (j0 >= lo && j0 + kTcTile <= hi) {
                                copy_word(smem_u32(&sh_vs[stage][lane]), word, from >= 0, bar);
                            } else {
                                const uint32_t w = from >= 0 ? __ldg(reinterpret_cast<const uint32_t *>(word)) : 0u;
                                sh_vs[stage][lane] = mend_scales(t, all, j0, w, suspects[u], lane, y == 0);
                                mbar_arrive(bar);
                            }
                        }
                        if (++stage == stages) { stage = 0; phase ^= 1u; }
                    }
                }
            }
            ++unit;
            next_unit(p, cur, part.places, piece_end);     // (while this one's last tiles are on their way)
            to_tiles(cur);
            if (cur.at < piece_end) next = find(cur, unit_part(p, cur, piece_end), 0);
        }
    } else if (warp == 1) {
        // ================================ S^T = K Q^T ================================
        int ks = 0;
        uint32_t k_phase = 0, k = 0, unit = 0;             // k: tiles done
        const uint32_t idesc = make_idesc_e4m3(G::kCols);
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            if (part.count == 0) { next_unit(p, cur, part.places, piece_end); continue; }
            const uint64_t q = make_smem_desc(base + G::kQAt + (unit & 1u) * G::kQ);
            wait(q_ready(unit & 1u), (unit >> 1) & 1u);
            for (int n = 0; n < part.count && ok; ++n, ++k) {
                const uint32_t b = k & 7u;
                wait(s_free(b), ((k >> 3) & 1u) ^ 1u);
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    wait(k_full(ks), k_phase);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t a = make_smem_desc(k_at(ks));
                    if (elect_one()) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)        // 32 features each (a descriptor counts 16 bytes)
                            umma_f8(s_at(b), a + 2 * c, q + (y * (G::kCols * 128) >> 4) + 2 * c, idesc, y + c > 0);
                        if (y + 1 == HB) umma_commit(s_full(b));
                        umma_commit(k_empty(ks));
                    }
                    __syncwarp();
                    if (++ks == G::kKStages) { ks = 0; k_phase ^= 1u; }
                }
            }
            ++unit;
            next_unit(p, cur, part.places, piece_end);
        }
    } else if (warp == 2) {
        // ================================ O^T += V^T P^T ================================
        int vs = 0;
        uint32_t v_phase = 0, k = 0, unit = 0;
        const uint32_t idesc = make_idesc(G::kCols) | (1u << 15) | (1u << 16);
        typedef TileAt<2, kApart> lay;
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            if (part.count == 0) { next_unit(p, cur, part.places, piece_end); continue; }
            for (int n = 0; n < part.count && ok; ++n, ++k) {
                const uint32_t x = k & 1u;
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    wait(v_full(vs), v_phase);
                    if (!ok) break;
                    if (y == 0) wait(p_ready(x), (k >> 1) & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t a = mn_desc(v_at(vs), lay::block, lay::group), b = p_desc<G::kPRow>(base + G::kPAt + x * G::kP);
                    const uint32_t d = o_at(unit & 1u, G::kSplit ? 0 : x) + y * G::kCols;
                    if (elect_one()) {
#pragma unroll
                        for (int c = 0; c < 8; ++c)        // 16 keys each
                            umma_bf16(d, a + (c * 2 * lay::group >> 4), b + (c * 16 * G::kPRow >> 4), idesc, n >= kStep || c > 0);
                        if (y + 1 == HB) umma_commit(pv_done(x));
                        umma_commit(v_empty(vs));
                        if (n + 1 == part.count && y + 1 == HB) umma_commit(acc_full(unit & 1u));
                    }
                    __syncwarp();
                    if ((vs ^= 1) == 0) v_phase ^= 1u;
                }
            }
            ++unit;
            next_unit(p, cur, part.places, piece_end);
        }
    } else if (warp < 12) {
        // ================================ softmax: a thread per key ================================
        const int x = (warp - 4) >> 2, wq = warp & 3, wt = wq * 32 + lane;
        const int bar_id = 1 + x;
        const int row0 = G::kSplit ? 8 * x : 0;            // of the warpgroup's rows: also their first column of S, P and the accumulator
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        const int p_sw = NR == 8 ? (wt >> 2) & 1 : (wt >> 1) & 3;
        const uint32_t p_row = base + G::kPAt + wt * G::kPRow, p_hi = (uint32_t)(((row0 / 8) ^ p_sw) << 4), p_lo = (uint32_t)(((row0 / 8 + NR / 8) ^ p_sw) << 4);
        uint32_t k0 = 0, unit = 0;
        float l[kR];
        while (cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { next_unit(p, cur, part.places, piece_end); continue; }
            const Tile t = cur.t;
            const Seen all = seen_by_all(p, t, cur.pre);
            const int u = unit & 1;
            const uint32_t o_tm = o_at(u, G::kSplit ? 0 : x) + lanes + row0;
            float *sh_m = sh_ms[u][x];
            if (unit >= 2) ok = bar_wait(unit_end(u), ((unit >> 1) - 1u) & 1u, abort_flag, ws) && ok;
#pragma unroll
            for (int r = 0; r < kR; ++r) l[r] = 0.f;
            const int n0 = G::kSplit ? 0 : (int)((k0 & 1u) ^ (uint32_t)x);         // this warpgroup's tiles: n0, n0 + kStep, ..
            if (n0 >= count && wt < kR) sh_m[wt] = kNone;
#pragma unroll 1
            for (int n = n0; n < count; n += kStep) {
                const uint32_t k = k0 + n, b = k & 7u;
                const uint32_t s_tm = s_at(b) + lanes + row0;
                ok = bar_wait(s_full(b), (k >> 3) & 1u, abort_flag, ws) && ok;
                __syncwarp();
                tc_fence_after();
                const float kf = q8_factor((sh_ks[b][wt >> 2] >> (8 * (wt & 3))) & 255u);
                const int j0 = key_tile(t, begin + n) * kTcTile, j = j0 + wt;
                const bool whole = j0 >= all.all_lo && j0 + kTcTile <= all.all_hi;
                uint32_t seen = 0;                         // by which rows, where not by all
                if (!whole) {
                    if (all.differ) {
#pragma unroll 1
                        for (int r = 0; r < kR; ++r) seen |= (uint32_t)sees(j, sh_hi[u][row0 + r], sh_lo[u][row0 + r], p.sinks) << r;
                    } else {
                        seen = sees(j, all.all_hi, all.all_lo, p.sinks) ? ~0u : 0u;
                    }
                }
                float s[kR];
                auto load = [&]() {                        // the key's scores, both parts of the queries
                    float v[2][8];
                    tmem_ld8_two(s_tm, s_tm + NR, v[0], v[1]);
#pragma unroll
                    for (int i = 0; i < kR; ++i) s[i] = fmaf(v[1][i], 0.0625f, v[0][i]);
                };
                auto hide = [&]() {                        // what a row does not see: -inf
                    if (!whole) {
#pragma unroll
                        for (int i = 0; i < kR; ++i) s[i] = (seen >> i) & 1u ? s[i] : -INFINITY;
                    }
                };
                auto against_max = [&]() {                 // exponents; rows and keys have their powers of two
#pragma unroll
                    for (int i = 0; i < kR; i += 4) {
                        const float4 m = *reinterpret_cast<const float4 *>(&sh_m[i]), f = *reinterpret_cast<const float4 *>(&sh_rf[u][row0 + i]);
                        s[i] = fmaf(s[i], f.x * kf, -m.x); s[i + 1] = fmaf(s[i + 1], f.y * kf, -m.y);
                        s[i + 2] = fmaf(s[i + 2], f.z * kf, -m.z); s[i + 3] = fmaf(s[i + 3], f.w * kf, -m.w);
                    }
                    hide();
                };
                bool grown = true;                         // (the warpgroup's first tile of the unit sets the maxima)
                if (n >= kStep) {
                    load();
                    against_max();
                    float top = s[0];
#pragma unroll
                    for (int i = 1; i < kR; ++i) top = fmaxf(top, s[i]);
                    grown = wg_any(bar_id, top > 8.f || !ok);
                }
                // the product of the tile before the last is done: its P may be overwritten (and, tiles in turn, the accumulator scaled)
                if (k >= 2) ok = bar_wait(pv_done(k & 1u), ((k >> 1) - 1u) & 1u, abort_flag, ws) && ok;
                if (__builtin_expect(grown, false)) {
                    // ---- some row's maximum has grown: new maxima, sums and accumulator brought to them
                    if (G::kSplit && n >= 1) ok = bar_wait(pv_done((k - 1) & 1u), ((k - 1) >> 1) & 1u, abort_flag, ws) && ok;
                    load();
#pragma unroll
                    for (int i = 0; i < kR; i += 4) {
                        const float4 f = *reinterpret_cast<const float4 *>(&sh_rf[u][row0 + i]);
                        s[i] *= f.x * kf; s[i + 1] *= f.y * kf; s[i + 2] *= f.z * kf; s[i + 3] *= f.w * kf;
                    }
                    hide();
                    {
                        const float top = reduce_rows<kR, true>(s, lane);
                        if (lane < kR) sh_wm[x][wq][lane] = top;
                    }
                    if (wg_any(bar_id, !ok)) { ok = false; break; }
                    if (wt < kR) {
                        const float top = fmaxf(fmaxf(sh_wm[x][0][wt], sh_wm[x][1][wt]), fmaxf(sh_wm[x][2][wt], sh_wm[x][3][wt]));
                        const float m = n < kStep ? kNone : sh_m[wt], nm = top > m + 8.f || (m == kNone && top > kNone) ? top : m;
                        sh_c[x][wt] = nm == m ? 1.f : ex2f(m - nm);
                        sh_m[wt] = nm;
                    }
                    wg_sync(bar_id);
                    if (n >= kStep) {
#pragma unroll
                        for (int r = 0; r < kR; r += 4) {
                            const float4 c = *reinterpret_cast<const float4 *>(&sh_c[x][r]);
                            l[r] *= c.x; l[r + 1] *= c.y; l[r + 2] *= c.z; l[r + 3] *= c.w;
                        }
                        tc_fence_after();
#pragma unroll 1
                        for (int y = 0; y < HB; ++y) {
                            float o[2][8];
                            tmem_ld8_two(o_tm + y * G::kCols, o_tm + y * G::kCols + NR, o[0], o[1]);
#pragma unroll
                            for (int z = 0; z < 2; ++z)
#pragma unroll
                                for (int i = 0; i < 8; ++i) o[z][i] *= sh_c[x][i];
                            tmem_st8(o_tm + y * G::kCols, o[0]);
                            tmem_st8(o_tm + y * G::kCols + NR, o[1]);
                        }
                        tmem_wait_st();
                    }
                    load();
                    against_max();
                }
                // ---- the scores have been read; probabilities of the key -> its row of P
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(s_free(b));
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = ex2f(s[2 * i]), b2 = ex2f(s[2 * i + 1]);
                    l[2 * i] += a;
                    l[2 * i + 1] += b2;
                    split_bf16(a, b2, hi[i], lo[i]);
                }
                const uint32_t to = p_row + (k & 1u) * G::kP;
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + p_hi), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + p_lo), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready(k & 1u));
            }
            // ---- the unit's end: sums over the warp's keys
            if (wg_any(bar_id, !ok)) break;
            const float sum = reduce_rows<kR, false>(l, lane);
            if (lane < kR) sh_wl[u][x][wq][lane] = sum;
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_full(u));
            k0 += (uint32_t)count;
            ++unit;
            next_unit(p, cur, part.places, piece_end);
        }
    } else if (warp >= 16) {
        // ================================ V: codes -> bf16 ================================
        constexpr int kGroups = G::kTurners / 4;           // a group of four warps takes every kGroups-th stage
        const int group = (warp - 16) >> 2, key0 = ((warp - 16) & 3) * 32;
        uint32_t i = (uint32_t)group, end = 0;             // stages
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const uint32_t begin = end;
            end += (uint32_t)part.count * HB;
#pragma unroll 1
            for (; i < end && ok; i += kGroups) {
                const uint32_t rs = i % G::kRawStages, vs = i & 1u;
                wait(raw_full(rs), (i / G::kRawStages) & 1u);
                wait(v_empty(vs), ((i >> 1) & 1u) ^ 1u);
                if (!ok) break;
                uint32_t scale[1] = {(sh_vs[rs][(key0 + lane) >> 2] >> (8 * (lane & 3))) & 255u};
                turn_stage<2, 1>(r_at(rs), v_at(vs), key0, min(p.D, 128), HB == 1 ? p.D : p.D - 128 * (int)((i - begin) & 1u), scale, lane);
                if (lane == 0) {
                    mbar_arrive(v_full(vs));
                    mbar_arrive(raw_empty(rs));
                }
            }
            next_unit(p, cur, part.places, piece_end);
        }
    } else {
        // ================================ queries, a unit ahead; units' ends ================================
        const int wq = warp & 3, wt = wq * 32 + lane;
        const int bar_id = 3;
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        uint32_t k0 = 0, unit = 0;
        auto queries = [&](const Cursor<NR, kTcTile> &c, int u) {      // (the unit before the last has ended here: all of it may be reused)
            load_query_parts<HB, NR>(p, c.start, c.h, c.t.r0, c.t.rows, base + G::kQAt + u * G::kQ, sh_rf[u], wt);
            if (wt < NR) {
                const int pos = c.pre + fast_div(c.t.r0 + min(wt, c.t.rows - 1), p.gdiv);
                sh_hi[u][wt] = p.mask == MRP_ATTN_CAUSAL ? pos + 1 : c.t.hi;
                sh_lo[u][wt] = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
            }
            mbar_arrive(q_ready(u));
        };
        to_tiles(cur);
        Cursor<NR, kTcTile> ahead = cur;
#pragma unroll 1
        for (int first = 1; cur.at < piece_end; first = 0) {
            if (!first) {
                cur = ahead;
                if (cur.at >= piece_end) break;
            }
            // (the first round loads the first unit's queries, every round the next one's)
#pragma unroll 1
            for (int y = first; y >= 0; --y) {
                if (y == 0) {
                    next_unit(p, ahead, unit_part(p, ahead, piece_end).places, piece_end);
                    to_tiles(ahead);
                }
                if (ahead.at < piece_end) queries(ahead, (unit + 1 - y) & 1);
            }
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            const Tile t = cur.t;
            const int u = unit & 1;
            ok = bar_wait(acc_full(u), (unit >> 1) & 1u, abort_flag, ws);
            if (wg_any(bar_id, !ok)) break;
            bool has[2];                               // tiles in turn: the warpgroup had one
#pragma unroll
            for (int y = 0; y < 2; ++y) has[y] = (int)((k0 & 1u) ^ (uint32_t)y) < count;
            tc_fence_after();
            const bool whole_unit = count == t.tiles;
            const int slot = 2 * (int)blockIdx.x + (begin == 0 ? 1 : 0);
            const int rows = t.rows;
            if (wt < NR) {
                float lw[2], mw[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int x = G::kSplit ? wt >> 3 : y;     // rows by halves: the row's warpgroup alone
                    lw[y] = sh_wl[u][x][0][wt & 7] + sh_wl[u][x][1][wt & 7] + sh_wl[u][x][2][wt & 7] + sh_wl[u][x][3][wt & 7];
                    mw[y] = sh_ms[u][x][wt & 7];
                }
                if (G::kSplit) lw[1] = 0.f;
                const float M = fmaxf(mw[0], mw[1]);
                const float f0 = mw[0] == M ? 1.f : ex2f(mw[0] - M), f1 = mw[1] == M ? 1.f : ex2f(mw[1] - M);
                const float L = lw[0] * f0 + lw[1] * f1;
                float inv = whole_unit ? inverse(L) : 1.f;
                // (the row's features, in a part of them too; its log-sum-exp knows nothing of values)
                if (suspects[u].n > 0 && suspects_hit(suspects[u], sh_hi[u][wt], sh_lo[u][wt], p.sinks)) inv = __int_as_float(0x7FC00000);
                sh_f[0][wt] = f0 * inv;
                sh_f[1][wt] = f1 * inv;
                if (wt < rows) {
                    const int rr = t.r0 + wt, tok = fast_div(rr, p.gdiv), head = cur.h * p.g + rr - tok * p.g;
                    if (!whole_unit) {
                        __stcg(p.part.ml + (size_t)slot * NR + wt, make_float2(M, L));
                    } else {
                        sh_out[wt] = (int64_t)(cur.start + tok) * p.out_stride + (int64_t)head * p.D;
                        if (p.lse) p.lse[(int64_t)(cur.start + tok) * p.H + head] = log_sum(M, L);
                    }
                }
            }
            wg_sync(bar_id);
#pragma unroll
            for (int y = 0; y < HB; ++y) {             // a thread per feature, of each 128
                const int f = y * 128 + wt;
                float a[NR];
#pragma unroll
                for (int i = 0; i < NR; ++i) a[i] = 0.f;
#pragma unroll
                for (int z = 0; z < (G::kSplit ? 1 : 2); ++z)
                    if (G::kSplit || has[z]) {
                        float o[2 * NR];
                        tmem_ld_n<2 * NR>(o_at(u, z) + y * G::kCols + lanes, o);
#pragma unroll
                        for (int i = 0; i < NR; ++i) a[i] = fmaf(o[i] + o[NR + i], sh_f[z][i], a[i]);
                    }
                if (f < p.D && whole_unit) {
#pragma unroll
                    for (int i = 0; i < NR; ++i)
                        if (i < rows) reinterpret_cast<__nv_bfloat16 *>(p.out)[sh_out[i] + f] = __float2bfloat16_rn(a[i]);
                } else if (f < p.D) {
                    float *to = p.part.o + (size_t)slot * NR * G::kWide + f;
#pragma unroll
                    for (int i = 0; i < NR; ++i)
                        if (i < rows) __stcg(to + i * G::kWide, a[i]);
                }
            }
            tc_fence_before();
            if (!whole_unit) {
                // ---- the pieces of the unit meet: the CTA that arrives last joins them in order
                int c0, c1;
                unit_pieces(p, cur, per, c0, c1);
                wg_sync(bar_id);
                if (wt == 0) sh_last = arrive_acq_rel(p.part.counters + c0) == c1 - c0;
                wg_sync(bar_id);
                if (sh_last) {
                    const JoinArgs ja = join_args(p, cur.start, cur.h, t.r0, rows, c0, c1);
                    join_rows<NR, G::kWide, 1, 4>(ja, wq, lane);          // (registers)
                    if (wt == 0) p.part.counters[c0] = 0;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(unit_end(u));
            wg_sync(bar_id);                           // sh_f, sh_out and sh_last are read
            k0 += (uint32_t)count;
            ++unit;
        }
        if (wt == 0)                                   // (units are left over only where a wait gave up)
            settle_arrivals(p, cur, per, piece_end, [&](const Cursor<NR, kTcTile> &, int c0, int c1) {
                if (arrive_acq_rel(p.part.counters + c0) == c1 - c0) p.part.counters[c0] = 0;
            });
    }

    __syncthreads();
    if (*abort_flag) {
        // a wait gave up: give copies still in flight time to land before the CTA leaves
        const long long t0 = clock64();
        while (clock64() - t0 < 200000) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)G::kTmem) : "memory");
    }
}

template <int HB, int NR>
cudaError_t few_q8_launch(Ctx *c, const AttnParams &p, const CUtensorMap &km, const CUtensorMap &vm, const PageBoxes &bx, cudaStream_t st)
{
    const int sms = c->sm_count < kKvMaxSm ? c->sm_count : kKvMaxSm;
    cudaError_t e = launch_k(kv_attention_few_q8_kernel<HB, NR>, dim3(sms), dim3(FewQ8Geo<HB, NR>::kThreads), FewQ8Geo<HB, NR>::kSmem, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p, km, vm, bx);
    c->launches = 1;
    return note_err(c, e, "kv_attention_few_q8_kernel");
}

}  // namespace

// box_rows: rows of a box; 8-bit pools of the geometry attached.  `swizzled`: as an operand, rows of 128 bytes; else raw.
bool codes_map(Ctx *c, CUtensorMap *map, const void *pool, int box_rows, bool swizzled)
{
    const mrp_kv_config &kv = c->kv;
    const cuuint64_t D = (cuuint64_t)kv.head_dim;
    const cuuint64_t dims[4] = {D, (cuuint64_t)kv.page_size, (cuuint64_t)kv.n_kv_heads, (cuuint64_t)kv.n_pages};
    const cuuint64_t strides[3] = {D, (cuuint64_t)kv.page_size * D, (cuuint64_t)kv.page_stride};
    const cuuint32_t box[4] = {(cuuint32_t)(swizzled || kv.head_dim > 128 ? 128 : kv.head_dim), (cuuint32_t)box_rows, 1, 1}, es[4] = {1, 1, 1, 1};
    return ((EncodeTiledFn)c->kv_encode)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(pool), dims, strides, box, es,
                                         CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HB, int NR> static cudaError_t few_q8_prepare()
{
    return cudaFuncSetAttribute(kv_attention_few_q8_kernel<HB, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewQ8Geo<HB, NR>::kSmem);
}
cudaError_t kv_few_q8_prepare()
{
    cudaError_t all[] = {few_q8_prepare<1, 8>(), few_q8_prepare<1, 16>(), few_q8_prepare<2, 8>(), few_q8_prepare<2, 16>()};
    for (cudaError_t one : all)
        if (one != cudaSuccess) return one;
    return cudaSuccess;
}

// Sequences of up to 16 rows (p.rows_above, p.rows_upto say which), mostly of up to 8 if `eight`; p.part is in place.
cudaError_t launch_few_q8(Ctx *c, AttnParams &p, int box_rows, bool eight, cudaStream_t st)
{
    CUtensorMap km, vm;
    if (!codes_map(c, &km, p.k, box_rows, true) || !codes_map(c, &vm, p.v, box_rows, false)) return note_err(c, cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    PageBoxes bx = {};
    bx.rows = box_rows;
    p.lead = 5;
    if (eight) return p.D <= 128 ? few_q8_launch<1, 8>(c, p, km, vm, bx, st) : few_q8_launch<2, 8>(c, p, km, vm, bx, st);
    return p.D <= 128 ? few_q8_launch<1, 16>(c, p, km, vm, bx, st) : few_q8_launch<2, 16>(c, p, km, vm, bx, st);
}

}  // namespace mrp

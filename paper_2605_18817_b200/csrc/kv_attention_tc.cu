// Attention over the pages of a key / value cache on the 5th-generation tensor cores: bf16, heads of up to 256 features, page
// sizes that are multiples of 8 rows (boxes of whole swizzled groups tile them).
//
// The mathematics are those of kv_attention.cu: running maximum (raised only by more than 2^8), probabilities and sums in
// fp32, one line of tiles cut into equal pieces, joined where a unit is cut.  Two kernels, both fed by TMA, page by page, into
// a ring of 128-byte-swizzled stages of a K or a V tile (128 keys), both with accumulators in tensor memory:
//
// kv_attention_few_kernel   up to 16 query rows per sequence and key head (decoding, blocks).  Transposed; see there.  Bound by
//                           memory: 64 ragged sequences of up to 8191 positions, 32 / 8 heads of 128: 165 us, 6.2 TB/s.
// kv_attention_tc_kernel    more: 128 query rows (row r = new token r / g, head r % g of the key head's group) on the lanes.
//   warp 0        K and V tiles                       warp 1   MMAs
//   8 NT warps    softmax, two threads a row, half its keys each: S from tensor memory, the maximum of the halves met through
//                 shared memory, P = exp2(scale S - m) as bf16 back into the columns S came in: O += P V takes it from there
//                 (and V as stored: its keys are the contraction, an MN-major operand).  The first half's product starts
//                 while the second half's probabilities are still on their way.
//   P is rounded to bf16 once, as an operand (2^-8 of each probability at most); the sum takes the unrounded values.  Hi + lo
//   parts would double the products that bound prompts.  Units of up to 16 rows, which the transposed kernel computes with both
//   parts, get both here too (NT = 1), so a sequence's precision does not depend on the others of its batch: lo takes the
//   columns of scores that have been read, and a second product.  24 blocks of 16, which have none: 67 -> 68 us.
//   NT = 2 (prompts): two row tiles share every K and V tile and take turns, one in the MMAs while the other is in the
//   exponentials.  Per pair of 128 x 128 tiles of 128 features the products take 2048 cycles, the exponentials alone 2048 of
//   the special function unit; measured 3600 (the softmax's chain of tensor-memory loads, maximum, exponentials, stores is what
//   does not overlap).  2 prompts of 2000 behind 5600 positions, 32 / 8 heads: 478 us, 1.0 PFLOP/s in a run of a few
//   milliseconds; 533 to 543 us, 0.88 PFLOP/s in one of seconds, under the power cap.  In short runs a thread per row took 40 us
//   more, exponentials by a polynomial on the FMA pipe for a part of the scores 10 to 30.
//   NT = 1 (17 to 128 rows, and batches too small to give two row tiles to all SMs): two S buffers instead, the next S is
//   computed while this one is exponentiated; 24 blocks of 32 tokens 78 us against 51 for the bytes.
//   Where a maximum grows, each warp of a pair rescales half of the accumulator's columns, and the pair meets before the first
//   product of the tile may start: that product adds to all columns.
//
// Other sources of K and V (LAY), same tiles and MMAs:
//   kPacked  rows beside the queries, no pages: 4 prompts of 600 to 4000 tokens, 32 / 8 heads: 437 us, 0.74 PFLOP/s.  Joining reads
//            the row and its log-sum-exp before it writes them.
//   kCodes   8 bits: TMA fetches codes into raw stages, and warps of their own (two beside two row tiles, four beside one) turn
//            codes times scales into bf16 stages of the ring, exactly.  Waits, lookups and cleaning are functions then: a loop of
//            every role has to stay in the instruction caches (inlined: prompt chunks 810 us).  2 chunks of 2000 behind 4000 to
//            6000 positions, 32 / 8 heads: 630 us, 0.71 PFLOP/s; a ring of three stages beside the raw ones and the turning's
//            issue slots (47 % busy against 39 %) are what 16 bits does not pay.  Four turning warps spill and give 625; a third
//            raw stage and rolled loops over half a row's scores give nothing.  12 blocks of 32: 55 us.
//
// Pages hold what they hold behind a sequence's end: scores of positions a row does not see are replaced before they are
// used, and V rows that no row of the tile sees are zeroed in shared memory before the product (0 * NaN).  A V row with
// an infinity or NaN that only some rows of a tile see (later tokens of a prompt) is zeroed too and makes the output of
// the rows that do see it NaN, all features, instead of that of the rows that do not.
#include "kv_tile.cuh"

namespace mrp {
namespace {

template <int NB, int NT, int LAY> struct TcGeo {
    typedef Blocks<NB> B;
    // 8 bits: raw stages (128 rows of up to 128 codes) beside the ring, and warps that turn them into stages of it
    static constexpr int kRawStage = LAY == kCodes ? B::kStageBytes / 2 : 0;
    static constexpr int kRawStages = LAY != kCodes ? 0 : B::DB == 1 ? 4 : NT == 1 && B::HB == 1 ? 3 : 2;
    static constexpr int kTurners = LAY != kCodes ? 0 : NT == 1 ? 4 : 2;           // (eight with one row tile: blocks of 32 55 -> 61 us)
    static constexpr int kStages = LAY == kCodes ? (B::DB == 1 ? 8 : B::HB == 2 || NT == 2 ? 3 : 4)
                                                 : B::DB == 1 ? 10 : B::HB == 2 || NT == 2 ? 4 : 5;
    static constexpr int kQTile = NB * 128 * 128;          // queries of a row tile
    static constexpr int kQ = NT * kQTile;
    static constexpr int kRing = kStages * B::kStageBytes;
    static constexpr int kRaw = kQ + kRing;
    static constexpr int kBars = kRaw + kRawStages * kRawStage;
    static constexpr int kSmem = kBars + 1024 + 1024;      // + alignment of the base
    static constexpr int kThreads = 64 + NT * 256 + kTurners * 32;
    static constexpr int kRows = NT * 128;
    static_assert(NT == 1 || NB <= 2, "tensor memory: two row tiles of accumulators of at most 128 features");
};

// ======================================================================================================================
// Few rows (decoding, blocks): everything transposed.  S^T = K Q^T puts the 128 keys of a tile on the tensor-memory lanes
// and the 16 query rows on the columns, O^T += V^T P^T the features on the lanes: the MMAs and the exponentials do the work of
// the rows there are, not of 128, and all 128 threads of a warpgroup have a key each.
//   warp 0   K and V tiles by TMA, as below        warp 1   MMAs        warps 2, 3   queries and what rows see, a unit ahead
//   warps 4-7, 8-11   two warpgroups that take tiles in turn, each with its own S buffer, maxima, sums and accumulator (no
//            exchange between them): a thread turns its key's scores into probabilities and stores them as a row of the
//            operand P [keys][rows] in shared memory, bf16 hi and lo columns side by side (2^-17 together: the second
//            product costs nothing that shows)
//   warps 12-15   the units' ends: both accumulators joined, rows or partial results written, pieces joined, while the others
//            are in the next unit (accumulators, sums and maxima of two units).  The first warpgroup did it before: 24 single
//            tokens 65 against 61 us, at 64 features 54 against 44
// The maximum in use is common to a warpgroup's 128 keys, so a tile needs to know only whether some score exceeds it by
// more than 2^8: one barrier with a vote.  Only then are the row maxima reduced (lanes, then warps) and the accumulator
// rescaled.  Sums stay per thread until the unit's end.  K and V are the only streams that count: memory bounds it (64 ragged
// single tokens 165 us against 158 for the bytes; 24 sequences of 200 to 6000 positions, one token 61 and four 64 against 48;
// one token behind 2047 positions, 16 heads: 13, of which the launch, the cut and the joining of 16 pieces are most).  Caches of
// one or two tiles are bound by a unit's chain instead, about 6 us an SM: 256 sequences of 20 to 300 positions 118 against 27.
template <int NB> struct FewGeo {
    typedef Blocks<NB> B;
    static constexpr int NR = kFewRows;
    static constexpr int kCols = 2 * NR;                   // columns of P and of an accumulator of 128 features: hi, lo
    static constexpr int kStages = B::DB == 2 ? 5 : 10;
    static constexpr int kRing = kStages * B::kStageBytes;
    static constexpr int kP = 128 * 128;                   // P of a warpgroup: 128 keys, rows of 128 bytes
    static constexpr int kQ = NB * NR * 128;               // queries of a unit, two of them
    static constexpr int kPAt = kRing, kQAt = kPAt + 2 * kP, kBars = kQAt + 2 * kQ;
    static constexpr int kSmem = kBars + 1024 + 1024;
    static constexpr int kTmem = B::HB == 2 ? 512 : 256;   // of which 2 NR + 4 HB kCols are used
    static constexpr int kThreads = 512;
    static constexpr int kWide = B::HB * 128;              // features of a row of partial results
};
template <int NB, int LAY>
__global__ void __launch_bounds__(512, 1)
kv_attention_few_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap kmap,
                        const __grid_constant__ CUtensorMap vmap, const PageBoxes bx)
{
    typedef FewGeo<NB> G;
    constexpr int DB = G::B::DB, HB = G::B::HB;
    constexpr int NR = kFewRows;
    typedef RowTile<NR, kTcTile> Tile;
    extern __shared__ unsigned char smem_raw[];
    __shared__ long long sh_find[G::kThreads / 32 + 2];
    __shared__ Suspects suspects[2];
    __shared__ int sh_hi[2][NR], sh_lo[2][NR];             // what a row sees: [lo, hi) and the first positions
    __shared__ __align__(16) float sh_ms[2][2][NR], sh_c[2][NR];   // maximum in use (unit, warpgroup), factor to it
    __shared__ float sh_wm[2][4][NR], sh_wl[2][2][4][NR];  // row maxima and (of a unit) sums of the warps
    __shared__ float sh_f[2][NR];                          // the unit's end: factors of the accumulators,
    __shared__ int64_t sh_out[NR];                         //   where the rows go
    __shared__ int sh_last;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t ring = base;
    const uint32_t bars = base + G::kBars;
    auto full_bar = [&](int s) { return bars + 8 * s; };
    auto empty_bar = [&](int s) { return bars + 8 * (16 + s); };
    auto s_full = [&](int x) { return bars + 8 * (32 + x); };
    auto p_ready = [&](int x) { return bars + 8 * (34 + x); };
    auto pv_done = [&](int x) { return bars + 8 * (36 + x); };
    auto q_ready = [&](int x) { return bars + 8 * (38 + x); };
    auto unit_end = [&](int x) { return bars + 8 * (40 + x); };    // the unit is written: everything of it may be reused
    auto acc_full = [&](int x) { return bars + 8 * (42 + x); };    // the unit's sums, maxima and accumulators are there
    unsigned char *gbars = smem_raw + (base - smem_u32(smem_raw)) + G::kBars;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(gbars + 8 * 44);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    const WaitStatus ws = {p.b.status, p.b.user_status};

    if (tid == 0) {
        for (int s = 0; s < G::kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            mbar_init(p_ready(x), 4);
            mbar_init(pv_done(x), 1);
            mbar_init(q_ready(x), 64);
            mbar_init(unit_end(x), 4);
            mbar_init(acc_full(x), 8);
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
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;    // S of the two warpgroups, then their accumulators of two units
    auto s_at = [&](int x) { return tmem + x * NR; };
    auto o_at = [&](int u, int x) { return tmem + 2 * NR + (2 * u + x) * HB * G::kCols; };       // (HB accumulators of 128 features)
    pdl_wait();
    pdl_trigger();

    Cursor<NR, kTcTile> cur;
    long long per;
    const long long len = p.b.n_seqs <= 128 ? find_piece_warp(p, cur, per, blockIdx.x == 0 && warp == 0)
                                            : find_piece<NR, kTcTile, G::kThreads>(p, cur, per, sh_find);
    if (len == 0) cur.at = 0;
    const long long piece_end = len > 0 ? cur.at + len : 0;

    if (warp == 0) {
        // ================================ K and V tiles ================================
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { leave_unit(p, cur, part.places, piece_end); continue; }
            auto fetch = [&](const PageRef &r, const CUtensorMap *map) {
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    ok = ok && __all_sync(0xffffffffu, mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, ws));
                    if (!ok) return;
                    fetch_tile<DB, LAY>(p, map, bx, r, cur.h, 128 * y, ring + stage * G::B::kStageBytes, full_bar(stage), lane);
                    if (++stage == G::kStages) { stage = 0; phase ^= 1u; }
                }
            };
            PageRef now = look_up<LAY>(p, bx, cur.t, begin, cur.s, cur.start, lane), next = now, then = now;
            if (count > 1) next = look_up<LAY>(p, bx, cur.t, begin + 1, cur.s, cur.start, lane);
            fetch(now, &kmap);
            for (int n = 0; n < count; ++n) {
                if (n + 2 < count) then = look_up<LAY>(p, bx, cur.t, begin + n + 2, cur.s, cur.start, lane);
                if (n + 1 < count) fetch(next, &kmap);
                fetch(now, &vmap);
                now = next;
                next = then;
            }
            leave_unit(p, cur, part.places, piece_end);
        }
    } else if (warp == 1) {
        // ================================ MMAs ================================
        int stage = 0;
        uint32_t phase = 0, k = 0, unit = 0;
        bool ok = true;
        const uint32_t idesc_s = make_idesc(NR), idesc_o = make_idesc(G::kCols) | (1u << 15) | (1u << 16);
        typedef TileAt<DB, LAY> lay;
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, ws)); };
        auto step = [&]() { if (++stage == G::kStages) { stage = 0; phase ^= 1u; } };
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { leave_unit(p, cur, part.places, piece_end); continue; }
            const Tile t = cur.t;
            const Seen all = seen_by_all(p, t, cur.pre);
            const uint32_t sq = base + G::kQAt + (unit & 1u) * G::kQ;
            wait(q_ready(unit & 1u), (unit >> 1) & 1u);
            if (!ok) break;
            Suspects &sus = suspects[unit & 1];            // (the unit before the last is written: see the query warps)
            if (lane == 0) sus.n = 0;
            __syncwarp();
            auto scores = [&](uint32_t kk) {               // S^T of tile kk from the stages at hand
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    wait(full_bar(stage), phase);
                    if (!ok) return;
                    tc_fence_after();
                    const uint32_t ks = ring + stage * G::B::kStageBytes, qs = sq + y * DB * (NR * 128);
                    if (elect_one()) {
#pragma unroll
                        for (int c = 0; c < 4 * DB; ++c)
                            umma_bf16(s_at(kk & 1u), k_desc(ks + (c >> 2) * lay::block + (c & 3) * 32, lay::group),
                                      make_smem_desc(qs + (c >> 2) * (NR * 128) + (c & 3) * 32), idesc_s, y + c > 0);
                        if (y + 1 == HB) umma_commit(s_full(kk & 1u));
                        umma_commit(empty_bar(stage));
                    }
                    __syncwarp();
                    step();
                }
            };
            scores(k);
            for (int n = 0; n < count && ok; ++n, ++k) {
                if (n + 1 < count) scores(k + 1);
                const uint32_t ps = base + G::kPAt + (k & 1u) * G::kP;
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    wait(full_bar(stage), phase);
                    if (!ok) break;
                    const uint32_t vs = ring + stage * G::B::kStageBytes;
                    clean_tile<DB, LAY>(t, all, key_tile(t, begin + n) * kTcTile, vs, sus, lane);
                    if (y == 0) wait(p_ready(k & 1u), (k >> 1) & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int c = 0; c < 8; ++c)        // (one block of features: the second 64 lanes repeat it)
                            umma_bf16(o_at(unit & 1u, k & 1u) + y * G::kCols, mn_desc(vs + c * 2 * lay::group, DB == 2 ? lay::block : 0, lay::group), mn_desc(ps + c * 2048, 0, 1024), idesc_o,
                                      n >= 2 || c > 0);
                        if (y + 1 == HB) umma_commit(pv_done(k & 1u));
                        umma_commit(empty_bar(stage));
                    }
                    __syncwarp();
                    step();
                }
            }
            ++unit;
            leave_unit(p, cur, part.places, piece_end);
        }
    } else if (warp < 4) {
        // ================================ queries, a unit ahead ================================
        uint32_t unit = 0;
        bool ok = true;
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            if (part.count == 0) { leave_unit(p, cur, part.places, piece_end); continue; }
            const Tile t = cur.t;
            const int u = unit & 1;
            if (unit >= 2) {
                ok = __all_sync(0xffffffffu, mbar_wait(unit_end(u), ((unit >> 1) - 1u) & 1u, abort_flag, ws));
                if (!ok) break;
            }
            load_queries<NB, NR, 64>(p, cur.start, cur.h, t.r0, t.rows, base + G::kQAt + u * G::kQ, tid - 64);
            for (int r = tid - 64; r < NR; r += 64) {
                const int pos = cur.pre + fast_div(t.r0 + min(r, t.rows - 1), p.gdiv);
                sh_hi[u][r] = p.mask == MRP_ATTN_CAUSAL ? pos + 1 : t.hi;
                sh_lo[u][r] = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
            }
            mbar_arrive(q_ready(u));
            ++unit;
            leave_unit(p, cur, part.places, piece_end);
        }
    } else if (warp < 12) {
        // ================================ softmax: a thread per key, two warpgroups in turn ================================
        const int x = (warp - 4) >> 2, wq = warp & 3, wt = wq * 32 + lane;
        const int bar_id = 1 + x;
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        const uint32_t s_tm = s_at(x) + lanes;
        const uint32_t p_row = base + G::kPAt + x * G::kP + wt * 128;
        uint32_t k0 = 0, unit = 0;
        const float sc = p.scale_log2;
        bool ok = true;
        float l[NR];
        while (cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { leave_unit(p, cur, part.places, piece_end); continue; }
            const Tile t = cur.t;
            const Seen all = seen_by_all(p, t, cur.pre);
            const int u = unit & 1;
            const uint32_t o_tm = o_at(u, x) + lanes;
            float *sh_m = sh_ms[u][x];
            if (unit >= 2) ok = mbar_wait(unit_end(u), ((unit >> 1) - 1u) & 1u, abort_flag, ws);
            if (wg_any(bar_id, !ok)) break;
            if (wt < NR) sh_m[wt] = kNone;
            wg_sync(bar_id);
#pragma unroll
            for (int r = 0; r < NR; ++r) l[r] = 0.f;
            const int n0 = (int)((k0 & 1u) ^ (uint32_t)x); // this warpgroup's tiles: n0, n0 + 2, ..
            for (int n = n0; n < count; n += 2) {
                const uint32_t k = k0 + n;
                ok = mbar_wait(s_full(x), (k >> 1) & 1u, abort_flag, ws);
                __syncwarp();
                tc_fence_after();
                const int j0 = key_tile(t, begin + n) * kTcTile, j = j0 + wt;
                const bool whole = j0 >= all.all_lo && j0 + kTcTile <= all.all_hi;
                uint32_t seen = 0;                         // by which rows, where not by all
                if (!whole) {
                    if (all.differ) {
#pragma unroll 1
                        for (int r = 0; r < NR; ++r) seen |= (uint32_t)sees(j, sh_hi[u][r], sh_lo[u][r], p.sinks) << r;
                    } else {
                        seen = sees(j, all.all_hi, all.all_lo, p.sinks) ? ~0u : 0u;
                    }
                }
                float s[NR];
                auto load = [&]() {                        // the key's scores; what a row does not see: -inf
                    tmem_ld_n<NR>(s_tm, s);
                    if (!whole) {
#pragma unroll
                        for (int i = 0; i < NR; ++i) s[i] = (seen >> i) & 1u ? s[i] : -INFINITY;
                    }
                };
                auto against_max = [&]() {                 // exponents
#pragma unroll
                    for (int i = 0; i < NR; i += 4) {
                        const float4 m = *reinterpret_cast<const float4 *>(&sh_m[i]);
                        s[i] = fmaf(s[i], sc, -m.x); s[i + 1] = fmaf(s[i + 1], sc, -m.y);
                        s[i + 2] = fmaf(s[i + 2], sc, -m.z); s[i + 3] = fmaf(s[i + 3], sc, -m.w);
                    }
                };
                bool grown = true;                         // (the warpgroup's first tile of the unit sets the maxima)
                if (n >= 2) {
                    load();
                    against_max();
                    float top = s[0];
#pragma unroll
                    for (int i = 1; i < NR; ++i) top = fmaxf(top, s[i]);
                    grown = wg_any(bar_id, top > 8.f || !ok);
                }
                if (grown) {
                    // ---- some row's maximum has grown: new maxima, sums and accumulator brought to them
                    if (wg_any(bar_id, !ok)) { ok = false; break; }
                    load();
#pragma unroll
                    for (int i = 0; i < NR; ++i) s[i] *= sc;
                    {
                        const float top = reduce_rows<NR, true>(s, lane);
                        if (lane < NR) sh_wm[x][wq][lane] = top;
                    }
                    wg_sync(bar_id);
                    if (wt < NR) {
                        const float top = fmaxf(fmaxf(sh_wm[x][0][wt], sh_wm[x][1][wt]), fmaxf(sh_wm[x][2][wt], sh_wm[x][3][wt]));
                        const float m = sh_m[wt], nm = top > m + 8.f || (m == kNone && top > kNone) ? top : m;
                        sh_c[x][wt] = nm == m ? 1.f : ex2f(m - nm);
                        sh_m[wt] = nm;
                    }
                    wg_sync(bar_id);
                    if (n >= 2) {
#pragma unroll
                        for (int r = 0; r < NR; r += 4) {
                            const float4 c = *reinterpret_cast<const float4 *>(&sh_c[x][r]);
                            l[r] *= c.x; l[r + 1] *= c.y; l[r + 2] *= c.z; l[r + 3] *= c.w;
                        }
                        // (the product of this warpgroup's last tile is done: S of this one came after it)
#pragma unroll 1
                        for (int r0 = 0; r0 < HB * G::kCols; r0 += 16) {
                            float o[16];
                            tmem_ld_n<16>(o_tm + r0, o);
                            uint32_t w[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * sh_c[x][(r0 + i) & (NR - 1)]);
                            tmem_st16(o_tm + r0, w);
                        }
                        tmem_wait_st();
                    }
                }
                // ---- probabilities of the key -> its row of P
                if (grown) {
                    load();
                    against_max();
                }
#pragma unroll
                for (int c = 0; c < NR / 8; ++c) {
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 8 * c + 2 * i;
                        const float a = ex2f(s[r]), b = ex2f(s[r + 1]);
                        l[r] += a;
                        l[r + 1] += b;
                        split_bf16(a, b, hi[i], lo[i]);
                    }
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(p_row + ((c ^ (wt & 7)) << 4)), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(p_row + (((c + NR / 8) ^ (wt & 7)) << 4)), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready(x));
            }
            if (!ok) break;
            // ---- the unit's end: sums over the warp's keys, the last product
            const float sum = reduce_rows<NR, false>(l, lane);
            if (lane < NR) sh_wl[u][x][wq][lane] = sum;
            if (n0 < count) {
                const uint32_t last = k0 + (uint32_t)(n0 + ((count - 1 - n0) & ~1));
                ok = mbar_wait(pv_done(x), (last >> 1) & 1u, abort_flag, ws);
            }
            if (wg_any(bar_id, !ok)) break;
            tc_fence_before();
            if (lane == 0) mbar_arrive(acc_full(u));
            k0 += (uint32_t)count;
            ++unit;
            leave_unit(p, cur, part.places, piece_end);
        }
    } else {
        // ================================ units' ends: both accumulators joined, written, pieces joined ================================
        const int wq = warp & 3, wt = wq * 32 + lane;
        const int bar_id = 3;
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        uint32_t k0 = 0, unit = 0;
        bool ok = true;
        while (cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { leave_unit(p, cur, part.places, piece_end); continue; }
            const Tile t = cur.t;
            const int u = unit & 1;
            ok = mbar_wait(acc_full(u), (unit >> 1) & 1u, abort_flag, ws);
            if (wg_any(bar_id, !ok)) break;
            bool has[2];
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
                    lw[y] = sh_wl[u][y][0][wt] + sh_wl[u][y][1][wt] + sh_wl[u][y][2][wt] + sh_wl[u][y][3][wt];
                    mw[y] = sh_ms[u][y][wt];
                }
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
                for (int z = 0; z < 2; ++z)
                    if (has[z]) {
                        float o[2][NR];
                        tmem_ld16_go(o_at(u, z) + y * G::kCols + lanes, o[0]);
                        tmem_ld16_go(o_at(u, z) + y * G::kCols + lanes + NR, o[1]);
                        tmem_wait_ld();
                        tmem_landed16(o[0]);
                        tmem_landed16(o[1]);
#pragma unroll
                        for (int i = 0; i < NR; ++i) a[i] = fmaf(o[0][i] + o[1][i], sh_f[z][i], a[i]);
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
                    if (rows <= 4) join_rows<NR, G::kWide, 1, 8>(ja, wq, lane);
                    else join_rows<NR, G::kWide, 2, 4>(ja, wq, lane);
                    if (wt == 0) p.part.counters[c0] = 0;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(unit_end(u));
            wg_sync(bar_id);                           // sh_f, sh_out and sh_last are read
            k0 += (uint32_t)count;
            ++unit;
            leave_unit(p, cur, part.places, piece_end);
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

// ======================================================================================================================
// Many rows: row tiles of 128 on the lanes, NT of them a unit.
template <int NB, int NT, int LAY>
__global__ void __launch_bounds__(TcGeo<NB, NT, LAY>::kThreads, 1)
kv_attention_tc_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap kmap,
                       const __grid_constant__ CUtensorMap vmap, const PageBoxes bx)
{
    typedef TcGeo<NB, NT, LAY> G;
    constexpr int DB = G::B::DB, HB = G::B::HB;
    constexpr int kRows = G::kRows;
    typedef RowTile<kRows, kTcTile> Tile;
    // With the warps that turn codes there are roles enough to overrun the instruction caches: what a loop does rarely stands outside
    // of it then (prompt chunk 830 -> 632 us; packed prompts, with a role less, 468 -> 494).
    constexpr bool kShort = LAY == kCodes;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Cursor<kRows, kTcTile> sh_cur;
    __shared__ long long sh_find[G::kThreads / 32 + 2];
    __shared__ Suspects suspects[2];
    __shared__ float sh_top[2][NT][2][128], sh_sum[NT][2][128];    // what the halves of a row tell each other
    __shared__ int sh_last[NT][4];
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sq = base, ring = base + G::kQ;
    // barriers
    const uint32_t bars = base + G::kBars;
    auto full_bar = [&](int s) { return bars + 8 * s; };
    auto empty_bar = [&](int s) { return bars + 8 * (16 + s); };
    auto s_full = [&](int x) { return bars + 8 * (32 + x); };
    auto p_ready = [&](int x) { return bars + 8 * (34 + x); };
    auto pv_done = [&](int x) { return bars + 8 * (36 + x); };
    auto q_ready = [&](int x) { return bars + 8 * (38 + x); };
    auto p_half = [&](int x) { return bars + 8 * (40 + x); };
    auto raw_full = [&](int s) { return bars + 8 * (48 + s); };    // 8 bits
    auto raw_empty = [&](int s) { return bars + 8 * (56 + s); };
    unsigned char *gbars = smem_raw + (base - smem_u32(smem_raw)) + G::kBars;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(gbars + 8 * 42);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_holder + 1);
    const WaitStatus ws = {p.b.status, p.b.user_status};

    if (tid == 0) {
        for (int s = 0; s < G::kStages; ++s) {
            mbar_init(full_bar(s), LAY == kCodes ? G::kTurners : 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int s = 0; s < G::kRawStages; ++s) {
            mbar_init(raw_full(s), 1);
            mbar_init(raw_empty(s), G::kTurners);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            mbar_init(p_ready(x), 4);
            mbar_init(p_half(x), 4);
            mbar_init(pv_done(x), 1);
            mbar_init(q_ready(x), 256);
        }
        *abort_flag = 0;
        prefetch_tmap(&kmap);
        prefetch_tmap(&vmap);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_holder)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (kShort && warp == 2) {
        pdl_wait();
        Cursor<kRows, kTcTile> c;
        long long full = 1;
        c.at = 0;
        const long long piece = cut_line<kRows>(p, c, full, blockIdx.x == 0);
        if (lane == 0) {
            sh_cur = c;
            sh_find[0] = piece;
            sh_find[1] = full;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;    // columns 0..255: two S buffers (P in their lower halves), 256..511: O per row tile
    pdl_wait();
    pdl_trigger();

    Cursor<kRows, kTcTile> cur;
    long long per, len;
    if constexpr (kShort) {
        cur = sh_cur;
        len = sh_find[0];
        per = sh_find[1];
    } else {
        len = p.b.n_seqs <= 128 ? find_piece_warp(p, cur, per, blockIdx.x == 0 && warp == 0) : find_piece<kRows, kTcTile, G::kThreads>(p, cur, per, sh_find);
    }
    if (len == 0) cur.at = 0;
    const long long piece_end = len > 0 ? cur.at + len : 0;
    auto hold = [](uint32_t bar, uint32_t parity, volatile int *flag, const WaitStatus &w) {
        if constexpr (kShort) return bar_wait(bar, parity, flag, w);
        else return mbar_wait(bar, parity, flag, w);
    };
    auto go_on = [&](Cursor<kRows, kTcTile> &c, int places) {
        if constexpr (kShort) next_unit(p, c, places, piece_end);
        else leave_unit(p, c, places, piece_end);
    };

    if (warp == 0) {
        // ================================ TMA producer ================================
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { go_on(cur, part.places); continue; }
            const Tile t = cur.t;
            auto fetch = [&](const PageRef &r, int which) {
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    ok = ok && __all_sync(0xffffffffu, hold(LAY == kCodes ? raw_empty(stage) : empty_bar(stage), phase ^ 1u, abort_flag, ws));
                    if (!ok) return;
                    if constexpr (LAY == kCodes)
                        fetch_codes(p, which ? &vmap : &kmap, bx, r, cur.h, 128 * y, min(p.D, 128), base + G::kRaw + stage * G::kRawStage, raw_full(stage), lane);
                    else
                        fetch_tile<DB, LAY>(p, which ? &vmap : &kmap, bx, r, cur.h, 128 * y, ring + stage * G::B::kStageBytes, full_bar(stage), lane);
                    if (++stage == (LAY == kCodes ? G::kRawStages : G::kStages)) { stage = 0; phase ^= 1u; }
                }
            };
            PageRef now = look_up<LAY>(p, bx, t, begin, cur.s, cur.start, lane), next = now, then = now;
            if (count > 1) next = look_up<LAY>(p, bx, t, begin + 1, cur.s, cur.start, lane);
            fetch(now, 0);
            for (int n = 0; n < count; ++n) {              // the order in which the MMA warp takes them
                if (n + 2 < count) then = look_up<LAY>(p, bx, t, begin + n + 2, cur.s, cur.start, lane);
                if (NT == 2) fetch(now, 1);
                if (n + 1 < count) fetch(next, 0);
                if (NT == 1) fetch(now, 1);
                now = next;
                next = then;
            }
            go_on(cur, part.places);
        }
    } else if (warp == 1) {
        // ================================ MMA issuer ================================
        int stage = 0;
        uint32_t phase = 0, k = 0, unit = 0;               // k: tiles done
        bool ok = true, two_parts = false;
        const uint32_t idesc_s = make_idesc(128), idesc_o = make_idesc(DB * 64) | (1u << 16);
        typedef TileAt<DB, LAY> lay;
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, hold(bar, parity, abort_flag, ws)); };
        auto step = [&]() { if (++stage == G::kStages) { stage = 0; phase ^= 1u; } };
        auto mma_s = [&](int x, int row_tile, uint32_t ks, int y) {        // S buffer x (+)= Q_row_tile K^T, features 128 y ..
            // (descriptors that are added to instead of made anew: the issue of an MMA is about as long as its work)
            const uint64_t qd = make_smem_desc(sq + row_tile * G::kQTile + y * G::B::kStageBytes), kd = k_desc(ks, lay::group);
            if (elect_one()) {
#pragma unroll
                for (int c = 0; c < 4 * DB; ++c) {
                    if constexpr (LAY >= kPacked)
                        umma_bf16(tmem + x * 128, qd + (((c >> 2) * (128 * 128) + (c & 3) * 32) >> 4), kd + (((c >> 2) * lay::block + (c & 3) * 32) >> 4), idesc_s, y + c > 0);
                    else
                    umma_bf16(tmem + x * 128, make_smem_desc(sq + row_tile * G::kQTile + y * G::B::kStageBytes + (c >> 2) * (128 * 128) + (c & 3) * 32),
                              k_desc(ks + (c >> 2) * lay::block + (c & 3) * 32, lay::group), idesc_s, y + c > 0);
                }
                if (y + 1 == HB) umma_commit(s_full(x));
            }
            __syncwarp();
        };
        // O_row_tile += P_x V, keys 16 c0 .. 16 c0 + 63, features 128 y ..
        auto mma_o = [&](int x, int row_tile, uint32_t vs, int y, int c0, bool first) {
            const uint64_t vd = mn_desc(vs + c0 * 2 * lay::group, lay::block, lay::group);
            if (elect_one()) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if constexpr (LAY >= kPacked)
                        umma_ts(tmem + 256 + (row_tile + y) * 128, tmem + x * 128 + c0 * 16 + c * 8, vd + (c * 2 * lay::group >> 4), idesc_o, !first || c0 + c > 0);
                    else
                    umma_ts(tmem + 256 + (row_tile + y) * 128, tmem + x * 128 + c0 * 16 + c * 8, mn_desc(vs + (c0 + c) * 2 * lay::group, lay::block, lay::group), idesc_o, !first || c0 + c > 0);
                if (two_parts) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        umma_ts(tmem + 256 + (row_tile + y) * 128, tmem + x * 128 + 32 + c0 * 16 + c * 8, mn_desc(vs + (c0 + c) * 2 * lay::group, lay::block, lay::group), idesc_o, 1);
                }
                if (c0 == 4 && y + 1 == HB) umma_commit(pv_done(x));
            }
            __syncwarp();
        };
        auto release = [&](int s) {
            if (elect_one()) umma_commit(empty_bar(s));
            __syncwarp();
        };
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { go_on(cur, part.places); continue; }
            const Tile t = cur.t;
            const Seen all = seen_by_all(p, t, cur.pre);
            two_parts = NT == 1 && LAY != kPacked && t.rows <= kFewRows;
            Suspects &sus = suspects[unit & 1];
            if (lane == 0) sus.n = 0;
            __syncwarp();
            const int fine_to = p.window > 0 ? 0 : all.differ ? min(t.hi, all.all_hi) : t.hi;      // tiles up to here hold nothing to clean
            auto clean = [&](int n, uint32_t vs) {
                const int j0 = key_tile(t, begin + n) * kTcTile;
                if constexpr (!kShort) clean_tile<DB, LAY>(t, all, j0, vs, sus, lane);
                else if (j0 + kTcTile > fine_to) clean_rarely<DB>(t, all, j0, vs, sus, lane);
            };
            auto at_stage = [&](int s) { return ring + s * G::B::kStageBytes; };
#pragma unroll
            for (int x = 0; x < NT; ++x) wait(q_ready(x), unit & 1u);
            auto first_scores = [&](int x0) {              // S of the tile whose K is next in the ring, for all row tiles
#pragma unroll
                for (int y = 0; y < HB; ++y) {
                    wait(full_bar(stage), phase);
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll
                    for (int x = 0; x < NT; ++x) mma_s(NT == 2 ? x : x0, x, at_stage(stage), y);
                    release(stage);
                    step();
                }
            };
            first_scores(k & 1u);
            for (int n = 0; n < count && ok; ++n, ++k) {
                if constexpr (NT == 2) {
                    const int sv = stage;
                    const uint32_t pv = phase;
                    step();
                    const int sk = stage;
                    const uint32_t pk = phase;
                    if (n + 1 < count) step();
                    wait(full_bar(sv), pv);
                    if (!ok) break;
                    clean(n, at_stage(sv));
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        wait(p_half(x), k & 1u);
                        if (!ok) break;
                        tc_fence_after();
                        mma_o(x, x, at_stage(sv), 0, 0, n == 0);
                        wait(p_ready(x), k & 1u);
                        if (n + 1 < count && x == 0) wait(full_bar(sk), pk);
                        if (!ok) break;
                        tc_fence_after();
                        mma_o(x, x, at_stage(sv), 0, 4, n == 0);
                        if (n + 1 < count) mma_s(x, x, at_stage(sk), 0);
                    }
                    if (!ok) break;
                    release(sv);
                    if (n + 1 < count) release(sk);
                } else {
                    if (n + 1 < count) first_scores((k + 1) & 1u);
                    int sv[HB];
#pragma unroll
                    for (int y = 0; y < HB; ++y) {
                        wait(full_bar(stage), phase);
                        if (!ok) break;
                        clean(n, at_stage(stage));
                        if (y == 0) wait(p_half(k & 1u), (k >> 1) & 1u);
                        if (!ok) break;
                        tc_fence_after();
                        sv[y] = stage;
                        mma_o(k & 1u, 0, at_stage(stage), y, 0, n == 0);
                        step();
                    }
                    wait(p_ready(k & 1u), (k >> 1) & 1u);
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int y = 0; y < HB; ++y) {
                        mma_o(k & 1u, 0, at_stage(sv[y]), y, 4, n == 0);
                        release(sv[y]);
                    }
                }
            }
            ++unit;
            go_on(cur, part.places);
        }
    } else if (LAY == kCodes && warp >= 2 + 8 * NT) {
        // ================================ 8 bits: raw stages -> stages of the ring ================================
        constexpr int KR = G::kTurners ? 4 / (G::kTurners ? G::kTurners : 1) : 1;                // of a stage, a warp has 32 KR keys
        const int key0 = (warp - (2 + 8 * NT)) * 32 * KR;
        int stage = 0, raw = 0;
        uint32_t phase = 0, raw_phase = 0;
        bool ok = true;
        while (ok && cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { go_on(cur, part.places); continue; }
            const Tile t = cur.t;
            auto find = [&](int n) { return find_keys<KR>(p, t, n < count, begin + n, cur.s, key0, lane); };
            auto turn = [&](const uint32_t (&bytes)[KR]) {
#pragma unroll 1
                for (int y = 0; y < HB; ++y) {
                    ok = ok && __all_sync(0xffffffffu, hold(raw_full(raw), raw_phase, abort_flag, ws));
                    ok = ok && __all_sync(0xffffffffu, hold(empty_bar(stage), phase ^ 1u, abort_flag, ws));
                    if (!ok) return;
                    turn_stage<DB, KR>(base + G::kRaw + raw * G::kRawStage, ring + stage * G::B::kStageBytes, key0, min(p.D, 128), p.D - 128 * y, bytes, lane);
                    if (lane == 0) {
                        mbar_arrive(full_bar(stage));
                        mbar_arrive(raw_empty(raw));
                    }
                    if (++stage == G::kStages) { stage = 0; phase ^= 1u; }
                    if (++raw == G::kRawStages) { raw = 0; raw_phase ^= 1u; }
                }
            };
            // scales a tile ahead of their use, their pages another tile
            uint32_t kn[KR], vn[KR], k1[KR], v1[KR], k2[KR], v2[KR];
            KeyPlaces<KR> at = find(0);
            load_scales(p, p.k_scale, at, cur.h, kn);
            load_scales(p, p.v_scale, at, cur.h, vn);
            at = find(1);
            load_scales(p, p.k_scale, at, cur.h, k1);
            load_scales(p, p.v_scale, at, cur.h, v1);
            at = find(2);
            turn(kn);
            for (int n = 0; n < count && ok; ++n) {        // the order in which the MMA warp takes them
                load_scales(p, p.k_scale, at, cur.h, k2);
                load_scales(p, p.v_scale, at, cur.h, v2);
                at = find(n + 3);
                if (NT == 2) turn(vn);
                if (n + 1 < count) turn(k1);
                if (NT == 1) turn(vn);
#pragma unroll
                for (int y = 0; y < KR; ++y) { vn[y] = v1[y]; k1[y] = k2[y]; v1[y] = v2[y]; }
            }
            go_on(cur, part.places);
        }
    } else {
        // ================================ softmax: two threads per row ================================
        const int group = (warp - 2) >> 2, x = group >> 1, half = group & 1;       // row tile, half of its keys
        const int wq = warp & 3, row = wq * 32 + lane;     // lane quarter of tensor memory, row of the row tile
        const int pair = 1 + x * 4 + wq;                   // barrier of the two warps that share 32 rows
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        const uint32_t o_tm = tmem + 256 + x * 128 + half * (NB * 32) + lanes;
        uint32_t k = 0, unit = 0;
        bool ok = true;
        const float sc = p.scale_log2;
        // P V of tile kk done.  A barrier may be one phase behind what is waited for, not two: with two S buffers the
        // softmax can finish a tile while the product before the last still runs, so each buffer has its own.
        auto wait_pv = [&](uint32_t kk) {
            return NT == 2 ? hold(pv_done(x), kk & 1u, abort_flag, ws) : hold(pv_done(kk & 1u), (kk >> 1) & 1u, abort_flag, ws);
        };
        while (cur.at < piece_end) {
            const UnitPart part = unit_part(p, cur, piece_end);
            const int begin = part.begin, count = part.count;
            if (count == 0) { go_on(cur, part.places); continue; }
            const Tile t = cur.t;
            const int rows = min(128, t.rows - x * 128);   // of this row tile (can be negative)
            const bool two_parts = NT == 1 && LAY != kPacked && t.rows <= kFewRows;
            // ---- queries -> shared memory (the S products of the unit before are done: its last S has been read)
            load_queries<NB, 128, 256>(p, cur.start, cur.h, t.r0 + x * 128, rows, sq + x * G::kQTile, half * 128 + row);
            mbar_arrive(q_ready(x));
            float prior = 0.f;                             // log-sum-exp to join with (both threads of the row, before either writes)
            // ---- what the row sees; what all rows of the warp see
            const bool live = row < rows, warp_live = wq * 32 < rows;
            int hi_r = 0, lo_r = 0;
            if (live) {
                const int pos = cur.pre + fast_div(t.r0 + x * 128 + row, p.gdiv);
                hi_r = p.mask == MRP_ATTN_CAUSAL ? pos + 1 : t.hi;
                lo_r = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
                if (LAY == kPacked && p.join) {
                    const int rr = t.r0 + x * 128 + row, tok = fast_div(rr, p.gdiv);
                    prior = p.lse[(int64_t)(cur.start + tok) * p.H + cur.h * p.g + rr - tok * p.g];
                }
            }
            int all_hi = 0, all_lo = 0;
            if (warp_live) {
                const int a = t.r0 + x * 128 + wq * 32, b = t.r0 + x * 128 + min(rows, wq * 32 + 32) - 1;
                all_hi = p.mask == MRP_ATTN_CAUSAL ? cur.pre + fast_div(a, p.gdiv) + 1 : t.hi;
                all_lo = p.window > 0 ? max(0, cur.pre + fast_div(b, p.gdiv) + 1 - p.window) : 0;
            }
            float m = -INFINITY, l = 0.f;
            for (int n = 0; n < count; ++n, ++k) {
                const int buf = NT == 2 ? x : (int)(k & 1u);
                const uint32_t s_tm = tmem + buf * 128 + half * 64 + lanes;        // this half's scores, then its P
                ok = hold(s_full(buf), NT == 2 ? k & 1u : (k >> 1) & 1u, abort_flag, ws);
                __syncwarp();
                tc_fence_after();
                if (!warp_live) {
                    if (any_of(pair, 64, !ok)) { ok = false; break; }
                } else {
                    // twice through the half row's scores, 32 at a time: the maximum, then the probabilities
                    const int j0 = key_tile(t, begin + n) * kTcTile + half * 64;
                    const bool whole = j0 >= all_lo && j0 + 64 <= all_hi;
                    auto hide = [&](float *s, int i0) {    // what the row does not see
                        const int j = j0 + i0;
                        const uint32_t seen = bit_range(lo_r - j, hi_r - j) | bit_range(0, min(p.sinks, hi_r) - j);
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[i] = (seen >> i) & 1u ? s[i] : -INFINITY;
                    };
                    float s[32], t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        tmem_ld32(s_tm + 32 * c, s);
                        tmem_wait_ld();
                        tmem_landed32(s);
                        if (!whole) hide(s, 32 * c);
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            t0 = fmaxf(fmaxf(t0, s[i]), s[i + 1]);
                            t1 = fmaxf(fmaxf(t1, s[i + 2]), s[i + 3]);
                        }
                    }
                    t0 = fmaxf(t0, t1) * sc;
                    sh_top[k & 1u][x][half][row] = t0;
                    tmem_ld32(s_tm, s);                    // (on its way while the halves meet)
                    if (any_of(pair, 64, !ok)) { ok = false; break; }
                    const float top = fmaxf(t0, sh_top[k & 1u][x][half ^ 1][row]);
                    const bool grow = top > m + 8.f;
                    tmem_wait_ld();
                    tmem_landed32(s);
                    if (__any_sync(0xffffffffu, grow)) {   // (the same in both warps)
                        const float nm = grow ? top : m;
                        const float c = m == nm ? 1.f : ex2f(m - nm);
                        if (n > 0) {                       // the accumulator of the tiles so far, half its columns each
                            ok = wait_pv(k - 1);
                            if (any_of(pair, 64, !ok)) { ok = false; break; }
                            tc_fence_after();
#pragma unroll 1
                            for (int f = 0; f < NB * 2; ++f) {
                                float o[16];
                                tmem_ld_n<16>(o_tm + 16 * f, o);
                                uint32_t w[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(o[i] * c);
                                tmem_st16(o_tm + 16 * f, w);
                            }
                            // The first half's product adds to ALL columns and waits for the first half's warps alone: both halves'
                            // columns are stored before either goes on.
                            tmem_wait_st();
                            tc_fence_before();
                            any_of(pair, 64, false);
                            tc_fence_after();
                        }
                        l *= c;
                        m = nm;
                    }
                    const float mm = m == -INFINITY ? 0.f : m;
                    float l0 = 0.f, l1 = 0.f;
                    auto exponentials = [&](int i, uint32_t &w, float &a, float &b) {
                        fma2(s[2 * i], s[2 * i + 1], sc, -mm);
                        a = ex2f(s[2 * i]);
                        b = ex2f(s[2 * i + 1]);
                        add2(l0, l1, a, b);
                        w = pack_bf16(a, b);
                    };
                    if (!two_parts) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            if (!whole) hide(s, 32 * c);
                            uint32_t w[16];
                            float a, b;
#pragma unroll
                            for (int i = 0; i < 16; ++i) exponentials(i, w[i], a, b);
                            if (c == 0) {                  // (the second 32 scores lie above the columns P goes to)
                                tmem_ld32(s_tm + 32, s);
                                tmem_st16(s_tm, w);
                                tmem_wait_ld();
                                tmem_landed32(s);
                            } else {
                                tmem_st16(s_tm + 16, w);
                            }
                        }
                    } else {
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {      // what the rounding leaves out goes where the second 32 scores were
                            if (!whole) hide(s, 32 * c);
                            uint32_t w[16], lo[16];
                            float a, b;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                exponentials(i, w[i], a, b);
                                lo[i] = pack_bf16(a - __uint_as_float(w[i] << 16), b - __uint_as_float(w[i] & 0xFFFF0000u));
                            }
                            tmem_st16(s_tm + 16 * c, w);
                            if (c == 0) {
                                tmem_ld32(s_tm + 32, s);
                                tmem_wait_ld();
                                tmem_landed32(s);
                            }
                            tmem_st16(s_tm + 32 + 16 * c, lo);
                        }
                    }
                    l += l0 + l1;
                    tmem_wait_st();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(half ? p_ready(buf) : p_half(buf));
            }
            if (!ok) break;
            // ---- the unit's end (or this piece's)
            sh_sum[x][half][row] = l;
            ok = wait_pv(k - 1);
            __syncwarp();
            if (any_of(pair, 64, !ok)) break;
            tc_fence_after();
            if (warp_live) {
                const float L = l + sh_sum[x][half ^ 1][row];
                const Suspects &sus = suspects[unit & 1];
                const bool hit = sus.n > 0 && suspects_hit(sus, hi_r, lo_r, p.sinks);      // NaN features; the log-sum-exp knows nothing of values
                const bool whole_unit = count == t.tiles;
                const int rr = t.r0 + x * 128 + row, tok = fast_div(rr, p.gdiv), head = cur.h * p.g + rr - tok * p.g;
                const int f0 = half * (NB * 32);           // this half's features
                __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + (int64_t)(cur.start + tok) * p.out_stride + (int64_t)head * p.D + f0;
                float *lse = p.lse && live && half == 0 ? p.lse + (int64_t)(cur.start + tok) * p.H + head : nullptr;
                auto put32 = [&](int f, float *o, float inv, float was) {  // 32 features from f0 + f; `was`: weight of the other pass's row
                    if (LAY == kPacked && p.join) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] *= inv;
                        inv = 1.f;
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            if (live && was != 0.f && f0 + f + i < p.D) {
                                const uint4 w = *reinterpret_cast<const uint4 *>(dst + f + i);
                                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                                for (int y = 0; y < 4; ++y) {
                                    o[i + 2 * y] = fmaf(__uint_as_float(u[y] << 16), was, o[i + 2 * y]);
                                    o[i + 2 * y + 1] = fmaf(__uint_as_float(u[y] & 0xFFFF0000u), was, o[i + 2 * y + 1]);
                                }
                            }
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        if (live && f0 + f + i < p.D)
                            *reinterpret_cast<uint4 *>(dst + f + i) =
                                make_uint4(pack_bf16(o[i] * inv, o[i + 1] * inv), pack_bf16(o[i + 2] * inv, o[i + 3] * inv),
                                           pack_bf16(o[i + 4] * inv, o[i + 5] * inv), pack_bf16(o[i + 6] * inv, o[i + 7] * inv));
                };
                const int slot = (2 * (int)blockIdx.x + (begin == 0 ? 1 : 0)) * NT + x;
                float4 *parts = reinterpret_cast<float4 *>(p.part.o);       // slot: [NB * 16][128 rows] float4
                float inv = inverse(L), was = 0.f, total = log_sum(m, L);
                if (LAY == kPacked && p.join) {
                    const JoinWith with = join_with(m, L, prior);
                    inv = with.a;
                    was = with.b;
                    total = with.lse;
                }
                if (whole_unit && lse) *lse = total;
                if (!whole_unit && live && half == 0) __stcg(p.part.ml + (size_t)slot * 128 + row, make_float2(m, L));
#pragma unroll 1
                for (int f = 0; f < NB; ++f) {
                    float o[32];
                    tmem_ld32(o_tm + 32 * f, o);
                    tmem_wait_ld();
                    tmem_landed32(o);
                    if (hit) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __int_as_float(0x7FC00000);
                    }
                    if (whole_unit) {
                        put32(32 * f, o, inv, was);
                    } else if (live) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            __stcg(parts + ((size_t)slot * (NB * 16) + f0 / 4 + f * 8 + i) * 128 + row, make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
                    }
                }
                tc_fence_before();
                if (!whole_unit) {
                    // ---- the pieces of these 32 rows meet: the pair that arrives last joins them in order
                    int c0, c1;
                    unit_pieces(p, cur, per, c0, c1);
                    int *counter = p.part.counters + (c0 * NT + x) * 4 + wq;
                    any_of(pair, 64, false);
                    if (half == 0 && lane == 0) sh_last[x][wq] = arrive_acq_rel(counter) == c1 - c0;
                    any_of(pair, 64, false);
                    if (sh_last[x][wq] && live) {
                        constexpr int U = NT == 1 && LAY != kCodes ? 2 : 1;      // pieces in flight (registers)
                        auto slot_of = [&](int c) { return (size_t)((2 * c + (c == c0)) * NT + x); };
#pragma unroll 1
                        for (int f = 0; f < NB; ++f) {
                            float M = -INFINITY, S = 0.f, o[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0.f;
#pragma unroll 1
                            for (int cb = c0; cb <= c1; cb += U) {
                                float2 ml[U];
                                float4 a[U][8];
#pragma unroll
                                for (int y = 0; y < U; ++y) {
                                    const size_t sl = slot_of(min(cb + y, c1));
                                    ml[y] = __ldcg(p.part.ml + sl * 128 + row);
#pragma unroll
                                    for (int i = 0; i < 8; ++i) a[y][i] = __ldcg(parts + (sl * (NB * 16) + f0 / 4 + f * 8 + i) * 128 + row);
                                }
#pragma unroll
                                for (int y = 0; y < U; ++y)
                                    if (cb + y <= c1) {
                                        const float nm = fmaxf(M, ml[y].x);
                                        const float e = M == nm ? 1.f : ex2f(M - nm), w = ml[y].x == nm ? 1.f : ex2f(ml[y].x - nm);
                                        M = nm;
                                        S = fmaf(w, ml[y].y, S * e);
#pragma unroll
                                        for (int i = 0; i < 8; ++i) {
                                            o[4 * i] = fmaf(w, a[y][i].x, o[4 * i] * e); o[4 * i + 1] = fmaf(w, a[y][i].y, o[4 * i + 1] * e);
                                            o[4 * i + 2] = fmaf(w, a[y][i].z, o[4 * i + 2] * e); o[4 * i + 3] = fmaf(w, a[y][i].w, o[4 * i + 3] * e);
                                        }
                                    }
                            }
                            if (LAY == kPacked && p.join) {
                                const JoinWith with = join_with(M, S, prior);
                                put32(32 * f, o, with.a, with.b);
                                if (f == 0 && lse) *lse = with.lse;
                            } else {
                                put32(32 * f, o, inverse(S), 0.f);
                                if (f == 0 && lse) *lse = log_sum(M, S);
                            }
                        }
                    }
                    if (half == 0 && lane == 0 && sh_last[x][wq]) *counter = 0;
                }
            }
            ++unit;
            go_on(cur, part.places);
        }
        if (half == 0 && lane == 0)                    // (units are left over only where a wait gave up)
            settle_arrivals(p, cur, per, piece_end, [&](const Cursor<kRows, kTcTile> &c, int c0, int c1) {
                if (x * 128 + wq * 32 >= c.t.rows) return;             // no row of these 32: nobody counts them
                int *counter = p.part.counters + (c0 * NT + x) * 4 + wq;
                if (arrive_acq_rel(counter) == c1 - c0) *counter = 0;
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
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

template <int NB, int NT, int LAY>
cudaError_t tc_prepare()
{
    return cudaFuncSetAttribute(kv_attention_tc_kernel<NB, NT, LAY>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcGeo<NB, NT, LAY>::kSmem);
}
template <int NB, int NT, int LAY>
cudaError_t tc_launch(Ctx *c, const AttnParams &p, const CUtensorMap &km, const CUtensorMap &vm, const PageBoxes &bx, cudaStream_t st)
{
    const int sms = c->sm_count < kKvMaxSm ? c->sm_count : kKvMaxSm;
    cudaError_t e = launch_k(kv_attention_tc_kernel<NB, NT, LAY>, dim3(sms), dim3(TcGeo<NB, NT, LAY>::kThreads), TcGeo<NB, NT, LAY>::kSmem, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p, km, vm, bx);
    c->launches = 1;
    return note_err(c, e, "kv_attention_tc_kernel");
}

template <int NB, int LAY>
cudaError_t few_prepare()
{
    return cudaFuncSetAttribute(kv_attention_few_kernel<NB, LAY>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewGeo<NB>::kSmem);
}
template <int NB, int LAY>
cudaError_t few_launch(Ctx *c, const AttnParams &p, const CUtensorMap &km, const CUtensorMap &vm, const PageBoxes &bx, cudaStream_t st)
{
    const int sms = c->sm_count < kKvMaxSm ? c->sm_count : kKvMaxSm;
    cudaError_t e = launch_k(kv_attention_few_kernel<NB, LAY>, dim3(sms), dim3(FewGeo<NB>::kThreads), FewGeo<NB>::kSmem, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p, km, vm, bx);
    c->launches = 1;
    return note_err(c, e, "kv_attention_few_kernel");
}

// Rows of a TMA box: the largest power of two, 8 to 128, that divides a page (a box is whole groups of 8 swizzled rows and
// never crosses a page); 0: none does.
int tc_box_rows(int page_size)
{
    for (int r = kTcTile; r >= 8; r /= 2)
        if (page_size % r == 0) return r;
    return 0;
}

PageBoxes page_boxes(const mrp_kv_config &kv, bool join)
{
    PageBoxes bx = {};
    bx.rows = tc_box_rows(kv.page_size);
    if (!join) return bx;
    const int64_t group = 8ll * kv.head_dim, in_all = (int64_t)kv.n_pages * (kv.page_stride / group);
    if (kv.head_dim % 128 == 0 && kv.page_stride % group == 0 && in_all < INT_MAX) {
        bx.page_groups = (int)(kv.page_stride / group);
        bx.head_groups = kv.page_size / 8;
        bx.groups = (int)in_all;
    }
    return bx;
}

bool page_map(Ctx *c, CUtensorMap *map, const void *pool, const PageBoxes &bx)
{
    const mrp_kv_config &kv = c->kv;
    const cuuint64_t D = (cuuint64_t)kv.head_dim;
    const cuuint64_t dims_apart[4] = {D, (cuuint64_t)kv.page_size, (cuuint64_t)kv.n_kv_heads, (cuuint64_t)kv.n_pages};
    const cuuint64_t strides_apart[3] = {D * 2, (cuuint64_t)kv.page_size * D * 2, (cuuint64_t)kv.page_stride * 2};
    const cuuint32_t box_apart[4] = {64, (cuuint32_t)bx.rows, 1, 1}, es[4] = {1, 1, 1, 1};
    const cuuint64_t dims_joined[4] = {64, 8, D / 64, (cuuint64_t)bx.groups};
    const cuuint64_t strides_joined[3] = {D * 2, 128, D * 16};
    const cuuint32_t box_joined[4] = {64, 8, 2, (cuuint32_t)bx.rows / 8};
    return ((EncodeTiledFn)c->kv_encode)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(pool), bx.groups ? dims_joined : dims_apart,
                                         bx.groups ? strides_joined : strides_apart, bx.groups ? box_joined : box_apart, es,
                                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool kv_tc_takes(const mrp_config &cfg, const mrp_kv_config &kv)
{
    // (strides of a tensor map: multiples of 16 bytes below 2^40; features beyond the head's read as zeros)
    return cfg.dtype == MRP_BF16 && kv.n_pages > 0 && tc_box_rows(kv.page_size) > 0 &&
           kv.page_stride < (1ll << 39) && (long long)kv.page_size * kv.head_dim < (1ll << 39) && !(cfg.flags & MRP_FLAG_FORCE_SIMT);
}

// some call on the geometry runs on large tiles (rows over each other need no pages)
bool kv_tc_any(const mrp_config &cfg, const mrp_kv_config &)
{
    return cfg.dtype == MRP_BF16 && !(cfg.flags & MRP_FLAG_FORCE_SIMT);
}

size_t kv_tc_workspace_bytes()
{
    return kKvCounterBytes + (size_t)2 * kKvMaxSm * 2 * 128 * (128 * 4 + 8);      // (or one row tile of 256 features)
}

cudaError_t kv_tc_attach(Ctx *c)
{
    c->kv_encode = nullptr;
    if (!kv_tc_any(c->cfg, c->kv)) return cudaSuccess;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
    if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) return e != cudaSuccess ? e : cudaErrorNotSupported;
    cudaError_t all[] = {few_prepare<1, kApart>(), few_prepare<2, kApart>(), few_prepare<4, kApart>(), few_prepare<2, kJoined>(), few_prepare<4, kJoined>(),
                         tc_prepare<1, 1, kApart>(), tc_prepare<2, 1, kApart>(), tc_prepare<4, 1, kApart>(), tc_prepare<2, 1, kJoined>(),
                         tc_prepare<4, 1, kJoined>(), tc_prepare<1, 2, kApart>(), tc_prepare<2, 2, kApart>(),
                         tc_prepare<1, 1, kPacked>(), tc_prepare<2, 1, kPacked>(), tc_prepare<4, 1, kPacked>(), tc_prepare<1, 2, kPacked>(),
                         tc_prepare<2, 2, kPacked>(),
                         tc_prepare<1, 1, kCodes>(), tc_prepare<2, 1, kCodes>(), tc_prepare<4, 1, kCodes>(), tc_prepare<1, 2, kCodes>(),
                         tc_prepare<2, 2, kCodes>()};
    for (cudaError_t one : all)
        if (one != cudaSuccess) return one;
    if ((e = kv_few_q8_prepare()) != cudaSuccess || (e = kv_short_prepare()) != cudaSuccess) return e;
    c->kv_encode = fn;
    return cudaSuccess;
}

static void place_parts(Ctx *c, AttnParams &p)
{
    const size_t slots = (size_t)2 * kKvMaxSm * 2;
    p.part.counters = (int32_t *)c->kv_ws;
    p.part.ml = (float2 *)(c->kv_ws + kKvCounterBytes);
    p.part.o = (float *)(c->kv_ws + kKvCounterBytes + slots * 128 * 8);
}
// as many units of two row tiles as SMs, as far as the host knows
static bool units_for_all(const Ctx *c, const AttnParams &p, const mrp_kv_batch &batch)
{
    return (long long)batch.n_seqs * p.Hk + (long long)batch.n_tokens * p.H / 256 > c->sm_count;
}

cudaError_t launch_paged_attention_tc(Ctx *c, AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st)
{
    place_parts(c, p);
    const long long rows = (long long)batch.max_new * p.g;
    const bool narrow = c->kv.head_dim <= 64, wide = c->kv.head_dim > 128;
    // Two row tiles share the stream of K and V where there are units for all SMs; with fewer the smaller units end sooner (512
    // tokens alone 28 against 27 us, 1024 44 against 36, 2048 74 against 78; 24 blocks of 33 behind 3000 102 against 120).
    const bool two = rows > 128 && !wide && units_for_all(c, p, batch);
    CUtensorMap km, vm;
    PageBoxes bx;
    auto maps = [&](bool join) {
        bx = page_boxes(c->kv, join);
        return page_map(c, &km, p.k, bx) && page_map(c, &vm, p.v, bx) ? cudaSuccess : note_err(c, cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    };
    // Pages of up to 32 rows joined: one token each of 24 sequences 76 against 66 us at 16 rows, 64 against 63 at 64; prompts are
    // bound by their products.
    const bool join = tc_box_rows(c->kv.page_size) <= 32;
    cudaError_t e = maps(join);
    if (e != cudaSuccess) return e;
    auto few = [&]() {
        p.lead = 2;                        // (24 single tokens 63, 61, 61 us at 1, 2, 3; 128 short caches 89, 86, 85)
        if (narrow) return few_launch<1, kApart>(c, p, km, vm, bx, st);
        if (bx.groups) return wide ? few_launch<4, kJoined>(c, p, km, vm, bx, st) : few_launch<2, kJoined>(c, p, km, vm, bx, st);
        return wide ? few_launch<4, kApart>(c, p, km, vm, bx, st) : few_launch<2, kApart>(c, p, km, vm, bx, st);
    };
    // Rows a unit: 16, 128 or 256.  24 sequences of 200 to 6000 cached positions, 8 key heads of 128: 16 rows 61 us on the
    // transposed kernel, 75 on the 128-row one (one token of one sequence: 12.6 against 24); a transposed one for 32 or 64 rows
    // took 95 and 113 against 78 and 80.
    if (rows <= kFewRows) return few();
    // Two row tiles leave sequences of up to 16 rows to the transposed kernel, in a launch of their own: they would fill a unit of
    // 256 rows each (48 single tokens and a prompt of 512: 132 against 108 us), and two row tiles have no registers for both
    // parts of P (prompts 470 -> 494 us with them).  Where there is no such sequence it costs 5 us (three prompts of 1000: 94 ->
    // 98; longer ones 470 -> 478, under the power cap nothing).  One row tile takes all sequences: a second launch costs more
    // than it saves (30 single tokens and two blocks of 32: 69 against 90 us; 12 and a prompt of 512 at 256 features: 85 against
    // 115; only beyond about 200 sequences it gains, 200 and ten blocks of 32: 277 against 249).
    int launches = 0;
    if (two) {
        p.rows_upto = kFewRows;
        if ((e = few()) != cudaSuccess) return e;
        launches = c->launches;
        p.rows_above = kFewRows;
        p.rows_upto = INT_MAX;
    }
    if (two && bx.groups && (e = maps(false)) != cudaSuccess) return e;
    // (what a unit costs besides its tiles, in tiles: three 1000- to 2000-token prompts 235, 181, 159, 153 us at 1, 2, 3, 4)
    p.lead = two ? 4 : 3;
    if (two) e = narrow ? tc_launch<1, 2, kApart>(c, p, km, vm, bx, st) : tc_launch<2, 2, kApart>(c, p, km, vm, bx, st);
    else if (narrow) e = tc_launch<1, 1, kApart>(c, p, km, vm, bx, st);
    else if (bx.groups) e = wide ? tc_launch<4, 1, kJoined>(c, p, km, vm, bx, st) : tc_launch<2, 1, kJoined>(c, p, km, vm, bx, st);
    else e = wide ? tc_launch<4, 1, kApart>(c, p, km, vm, bx, st) : tc_launch<2, 1, kApart>(c, p, km, vm, bx, st);
    c->launches += launches;
    return e;
}

// ---- pages of 8 bits, rows beside the queries ---------------------------------------------------------------------------
bool kv_tc_takes_q8(const mrp_config &cfg, const mrp_kv_config &kv)
{
    // (a box is whole 16-byte runs of a row's codes, strides are multiples of 16 bytes)
    return kv_tc_any(cfg, kv) && kv.n_pages > 0 && tc_box_rows(kv.page_size) > 0 && kv.head_dim % 16 == 0 && kv.page_stride % 16 == 0 &&
           kv.page_stride < (1ll << 40) && (long long)kv.page_size * kv.head_dim < (1ll << 40);
}

cudaError_t launch_paged_attention_q8_tc(Ctx *c, AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st)
{
    place_parts(c, p);
    const mrp_kv_config &kv = c->kv;
    const long long rows = (long long)batch.max_new * p.g;
    const bool narrow = kv.head_dim <= 64, wide = kv.head_dim > 128;
    const bool two = rows > 128 && !wide && units_for_all(c, p, batch);
    PageBoxes bx = {};
    bx.rows = tc_box_rows(kv.page_size);
    if (rows <= kFewRows) return launch_few_q8(c, p, bx.rows, rows <= 8, st);
    CUtensorMap km, vm;
    if (!codes_map(c, &km, p.k, bx.rows, false) || !codes_map(c, &vm, p.v, bx.rows, false)) return note_err(c, cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    cudaError_t e;
    int launches = 0;
    auto one = [&]() {
        p.lead = 3;
        return narrow ? tc_launch<1, 1, kCodes>(c, p, km, vm, bx, st) : wide ? tc_launch<4, 1, kCodes>(c, p, km, vm, bx, st) : tc_launch<2, 1, kCodes>(c, p, km, vm, bx, st);
    };
    if (two) {
        p.rows_upto = kFewRows;
        if ((e = launch_few_q8(c, p, bx.rows, p.g <= 8, st)) != cudaSuccess) return e;
        launches = c->launches;
        p.rows_above = kFewRows;
        p.rows_upto = INT_MAX;
        p.lead = 4;
        e = narrow ? tc_launch<1, 2, kCodes>(c, p, km, vm, bx, st) : tc_launch<2, 2, kCodes>(c, p, km, vm, bx, st);
    } else {
        e = one();
    }
    c->launches += launches;
    return e;
}

bool kv_tc_takes_rows(const mrp_config &cfg, const mrp_kv_config &kv, const mrp_packed_kv &rows)
{
    return kv_tc_any(cfg, kv) && rows.k_stride < (1ll << 39) && rows.v_stride < (1ll << 39);
}

cudaError_t launch_packed_attention_tc(Ctx *c, AttnParams &p, const mrp_kv_batch &batch, cudaStream_t st)
{
    place_parts(c, p);
    const bool narrow = p.D <= 64, wide = p.D > 128;
    const bool two = (long long)batch.max_new * p.g > 128 && !wide && units_for_all(c, p, batch);
    PageBoxes bx = {};
    bx.rows = kTcTile;
    CUtensorMap km, vm;
    const void *ptr[2] = {p.k, p.v};
    const int64_t stride[2] = {p.k_stride, p.v_stride};
    for (int i = 0; i < 2; ++i) {
        const cuuint64_t dims[4] = {(cuuint64_t)p.D, (cuuint64_t)batch.n_tokens, (cuuint64_t)p.Hk, 1};
        const cuuint64_t strides[3] = {(cuuint64_t)stride[i] * 2, (cuuint64_t)p.D * 2, (cuuint64_t)stride[i] * 2};
        const cuuint32_t box[4] = {64, (cuuint32_t)bx.rows, 1, 1}, es[4] = {1, 1, 1, 1};
        if (((EncodeTiledFn)c->kv_encode)(i ? &vm : &km, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(ptr[i]), dims, strides, box, es,
                                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return note_err(c, cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    }
    p.lead = two ? 4 : 3;
    if (two) return narrow ? tc_launch<1, 2, kPacked>(c, p, km, vm, bx, st) : tc_launch<2, 2, kPacked>(c, p, km, vm, bx, st);
    return narrow ? tc_launch<1, 1, kPacked>(c, p, km, vm, bx, st) : wide ? tc_launch<4, 1, kPacked>(c, p, km, vm, bx, st) : tc_launch<2, 1, kPacked>(c, p, km, vm, bx, st);
}

}  // namespace mrp

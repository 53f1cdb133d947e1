// Attention over the pages of a key / value cache on the 5th-generation tensor cores: blocks and prompts, that is more
// query rows per sequence and key head than a 16-row tile holds (bf16, heads of up to 128 features, page sizes that TMA
// boxes tile).
//
// The mathematics are those of kv_attention.cu; here S = Q K^T and O += P V run as tcgen05.mma with 128 query rows
// (row r = new token r / g, head r % g of the key head's group) against tiles of 128 keys:
//   warp 0        fetches K and V tiles, page by page, by TMA into a ring of 128-byte-swizzled stages
//   warp 1        issues the MMAs: S into tensor memory, O += P V with P read from tensor memory (it lies in the columns
//                 S came in) and V as stored (its keys are the contraction: an MN-major operand)
//   4 NT warps    a warpgroup per 128 rows, a thread per row: S from tensor memory, running maximum and sum with no
//                 exchange between lanes, P = exp2(scale S - m) rounded to bf16 back into tensor memory, O at the end
// NT = 2 (prompts): two row tiles share every K and V tile and take turns, one in the MMAs while the other is in the
// exponentials; at 128 features both take about 1024 cycles per 128 x 128 tile, so neither waits long.  NT = 1 (blocks):
// two S buffers instead, the next S is computed while this one is exponentiated; the K / V stream bounds it.
// The accumulator stays in tensor memory; it is rescaled only when a row's maximum has grown by more than 2^8 over the
// one in use.  Tiles of all units form one line cut into equal pieces as in kv_attention.cu; a unit cut in two is joined
// row by row by the warp that arrives last.
//
// Pages hold what they hold behind a sequence's end: scores of positions a row does not see are replaced before they are
// used, and V rows that no row of the tile sees are zeroed in shared memory before the product (0 * NaN).  A V row with
// an infinity or NaN that only some rows of a tile see (later tokens of a prompt) is zeroed too and makes the output of
// the rows that do see it NaN, all features, instead of that of the rows that do not.
#include "kv_attention.cuh"
#include "tc_common.cuh"

namespace mrp {
namespace {

constexpr int kTcTile = 128;               // keys of a tile, rows of a row tile
constexpr int kMaxSuspects = 16;           // boundary tiles of a unit that are remembered for values that are not finite

struct WaitStatus {
    int32_t *status, *user_status;
};

template <int DB, int NT> struct TcGeo {   // DB: 64-feature blocks of a head
    static constexpr int kTileBytes = DB * 128 * 128;
    static constexpr int kStages = DB == 2 ? (NT == 2 ? 5 : 6) : 10;
    static constexpr int kQ = NT * kTileBytes;
    static constexpr int kRing = kStages * kTileBytes;
    static constexpr int kBars = kQ + kRing;
    static constexpr int kSmem = kBars + 1024 + 1024;      // + alignment of the base
    static constexpr int kThreads = 128 + NT * 128;
    static constexpr int kRows = NT * 128;
};

struct Suspects {                          // boundary tiles with V rows that were zeroed for what they held
    int n;
    int base[kMaxSuspects];
    uint32_t keys[kMaxSuspects][4];
};

__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], bf16
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t db, uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(db), "r"(idesc), "r"(acc) : "memory");
}
// 32 columns of the warp's 32 lanes; no wait
__device__ __forceinline__ void tmem_ld32(uint32_t a, float *v)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t a, const float *v)
{
    const uint32_t *r = reinterpret_cast<const uint32_t *>(v);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(a), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// Behind the wait: the compiler sees no other tie between the wait and the registers the loads fill, and may use them early.
__device__ __forceinline__ void tmem_landed32(float *v)
{
    asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                     "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                     "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                     "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]) :: "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// V as the B operand of P V: [keys][64 features] rows of 128 bytes, swizzled in groups of 8 keys.  The contraction (keys)
// runs down the rows, so the operand is MN-major: groups of 8 keys 1024 bytes apart, 64-feature blocks a tile apart.
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)((128 * 128) >> 4) << 16;               // next 64 features
    d |= (uint64_t)(1024 >> 4) << 32;                      // next 8 keys
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

template <int DB, int NT>
__global__ void __launch_bounds__(TcGeo<DB, NT>::kThreads, 1)
kv_attention_tc_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap kmap,
                       const __grid_constant__ CUtensorMap vmap, int box_rows)
{
    typedef TcGeo<DB, NT> G;
    constexpr int kRows = G::kRows;
    typedef RowTile<kRows, kTcTile> Tile;
    extern __shared__ unsigned char smem_raw[];
    __shared__ long long sh_find[G::kThreads / 32 + 2];
    __shared__ Suspects suspects[2];
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
    unsigned char *gbars = smem_raw + (base - smem_u32(smem_raw)) + G::kBars;
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(gbars + 8 * 40);
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
            mbar_init(q_ready(x), 128);
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
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;    // columns 0..255: two S buffers (P in their lower halves), 256..511: O per row tile
    pdl_wait();
    pdl_trigger();

    Cursor<kRows, kTcTile> cur;
    long long per;
    const long long len = find_piece<kRows, kTcTile, G::kThreads>(p, cur, per, sh_find);
    const long long piece_end = len > 0 ? cur.at + len : 0;
    long long at = len > 0 ? cur.at : 0;
    // (all roles walk the same units; a unit of the piece: tiles begin .. begin + count - 1 of cur.t)
    auto next_unit = [&](int count) {
        at += count;
        if (at < piece_end) {
            cur.i = cur.t.tiles - 1;
            cur.at = at - 1;
            advance(p, cur);
        }
    };

    if (warp == 0) {
        // ================================ TMA producer ================================
        int stage = 0;
        uint32_t phase = 0;
        const int pages = kTcTile / box_rows;              // boxes of a tile
        const int P = p.b.page.d;
        bool ok = true;
        while (ok && at < piece_end) {
            const int begin = cur.i, count = (int)min((long long)(cur.t.tiles - cur.i), piece_end - at);
            const Tile t = cur.t;
            // one tile of K (which = 0) or V, the pages of its visible positions
            auto fetch = [&](int n, int which) {
                if (!ok) return;
                ok = __all_sync(0xffffffffu, mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, ws));
                if (!ok) return;
                const int j0 = key_tile(t, begin + n) * kTcTile, j = j0 + lane * box_rows;
                const bool need = lane < pages && ((j < t.hi && j + box_rows > t.lo) || j < t.s1);
                int entry = 0, row = 0;
                if (need) {
                    const int pg = fast_div(j, p.b.page);
                    row = j - pg * P;
                    entry = __ldg(p.b.page_table + (size_t)cur.s * p.b.max_pages + pg);
                    if ((unsigned)entry >= (unsigned)p.b.n_pages) {
                        kv_bad_index(p.b);
                        entry = p.b.n_pages;               // outside the map: zeros arrive
                    }
                }
                const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, need));
                if (lane == 0) mbar_expect_tx(full_bar(stage), boxes * box_rows * 128u * DB);
                __syncwarp();
                if (need) {
                    const uint32_t dst = ring + stage * G::kTileBytes + lane * box_rows * 128;
#pragma unroll
                    for (int x = 0; x < DB; ++x)
                        tma_load_page(dst + x * (128 * 128), which ? &vmap : &kmap, 64 * x, row, cur.h, entry, full_bar(stage));
                }
                if (++stage == G::kStages) { stage = 0; phase ^= 1u; }
            };
            fetch(0, 0);
            for (int n = 0; n < count; ++n) {              // the order in which the MMA warp takes them
                if (NT == 2) fetch(n, 1);
                if (n + 1 < count) fetch(n + 1, 0);
                if (NT == 1) fetch(n, 1);
            }
            next_unit(count);
        }
    } else if (warp == 1) {
        // ================================ MMA issuer ================================
        int stage = 0;
        uint32_t phase = 0, k = 0, unit = 0;               // k: tiles done
        bool ok = true;
        const uint32_t idesc_s = make_idesc(128), idesc_o = make_idesc(DB * 64) | (1u << 16);
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, ws)); };
        auto step = [&]() { if (++stage == G::kStages) { stage = 0; phase ^= 1u; } };
        auto mma_s = [&](int x, int row_tile, uint32_t ks) {       // S buffer x = Q_row_tile K^T
            if (elect_one()) {
#pragma unroll
                for (int c = 0; c < 4 * DB; ++c) {
                    const uint32_t off = (c >> 2) * (128 * 128) + (c & 3) * 32;
                    umma_bf16(tmem + x * 128, make_smem_desc(sq + row_tile * G::kTileBytes + off), make_smem_desc(ks + off), idesc_s, c > 0);
                }
                umma_commit(s_full(x));
            }
            __syncwarp();
        };
        auto mma_o = [&](int x, int row_tile, uint32_t vs, bool first) {   // O_row_tile += P_x V
            if (elect_one()) {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    umma_ts(tmem + 256 + row_tile * 128, tmem + x * 128 + c * 8, v_desc(vs + c * 2048), idesc_o, !first || c > 0);
                umma_commit(pv_done(x));
            }
            __syncwarp();
        };
        auto release = [&](int s) {
            if (elect_one()) umma_commit(empty_bar(s));
            __syncwarp();
        };
        while (ok && at < piece_end) {
            const int begin = cur.i, count = (int)min((long long)(cur.t.tiles - cur.i), piece_end - at);
            const Tile t = cur.t;
            const int i0 = t.r0 / p.g, i1 = (t.r0 + t.rows - 1) / p.g;
            const bool differ = i0 != i1 && (p.mask == MRP_ATTN_CAUSAL || p.window > 0);
            const int all_hi = p.mask == MRP_ATTN_CAUSAL ? cur.pre + i0 + 1 : t.hi;
            const int all_lo = p.window > 0 ? max(0, cur.pre + i1 + 1 - p.window) : 0;
            Suspects &sus = suspects[unit & 1];
            if (lane == 0) sus.n = 0;
            __syncwarp();
            // V rows no row sees -> zeros; rows some see that hold what is not finite -> zeros, remembered
            auto clean = [&](int n, uint32_t vs) {
                const int j0 = key_tile(t, begin + n) * kTcTile;
                if ((j0 >= t.lo && j0 + kTcTile <= t.hi) || j0 + kTcTile <= t.s1) {
                    if (!differ || (j0 >= all_lo && j0 + kTcTile <= all_hi)) return;
                }
                uint32_t found[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int row = w * 32 + lane, j = j0 + row;
                    const bool seen = j < t.hi && (j >= t.lo || j < t.s1);
                    bool bad = false;
                    if (seen && differ && !(j >= all_lo && j < all_hi)) {
                        for (int c = 0; c < 8 * DB; ++c) {
                            uint32_t u[4];
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                                         : "r"(vs + (c >> 3) * (128 * 128) + row * 128 + (((c + lane) & 7) << 4)) : "memory");
#pragma unroll
                            for (int y = 0; y < 4; ++y) bad |= (u[y] & 0x7F800000u) == 0x7F800000u || (u[y] & 0x7F80u) == 0x7F80u;
                        }
                    }
                    found[w] = __ballot_sync(0xffffffffu, bad);
                    if (!seen || bad)
                        for (int c = 0; c < 8 * DB; ++c)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};"
                                         ::"r"(vs + (c >> 3) * (128 * 128) + row * 128 + (((c + lane) & 7) << 4)), "r"(0u) : "memory");
                }
                if (lane == 0 && (found[0] | found[1] | found[2] | found[3])) {
                    const int at_n = sus.n;
                    if (at_n < kMaxSuspects) {
                        sus.base[at_n] = j0;
#pragma unroll
                        for (int w = 0; w < 4; ++w) sus.keys[at_n][w] = found[w];
                    }
                    sus.n = at_n + 1;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            };
#pragma unroll
            for (int x = 0; x < NT; ++x) wait(q_ready(x), unit & 1u);
            wait(full_bar(stage), phase);
            if (!ok) break;
            tc_fence_after();
            if constexpr (NT == 2) {
                mma_s(0, 0, ring + stage * G::kTileBytes);
                mma_s(1, 1, ring + stage * G::kTileBytes);
            } else {
                mma_s(k & 1u, 0, ring + stage * G::kTileBytes);
            }
            release(stage);
            step();
            for (int n = 0; n < count && ok; ++n, ++k) {
                if constexpr (NT == 2) {
                    const int sv = stage;
                    const uint32_t pv = phase;
                    step();
                    const int sk = stage;
                    const uint32_t pk = phase;
                    if (n + 1 < count) step();
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        wait(p_ready(x), k & 1u);
                        if (x == 0) {
                            wait(full_bar(sv), pv);
                            if (!ok) break;
                            clean(n, ring + sv * G::kTileBytes);
                        }
                        if (!ok) break;
                        tc_fence_after();
                        mma_o(x, x, ring + sv * G::kTileBytes, n == 0);
                        if (n + 1 < count) {
                            if (x == 0) wait(full_bar(sk), pk);
                            if (!ok) break;
                            mma_s(x, x, ring + sk * G::kTileBytes);
                        }
                    }
                    if (!ok) break;
                    release(sv);
                    if (n + 1 < count) release(sk);
                } else {
                    if (n + 1 < count) {
                        wait(full_bar(stage), phase);
                        if (!ok) break;
                        mma_s((k + 1) & 1u, 0, ring + stage * G::kTileBytes);
                        release(stage);
                        step();
                    }
                    wait(p_ready(k & 1u), (k >> 1) & 1u);
                    wait(full_bar(stage), phase);
                    if (!ok) break;
                    clean(n, ring + stage * G::kTileBytes);
                    tc_fence_after();
                    mma_o(k & 1u, 0, ring + stage * G::kTileBytes, n == 0);
                    release(stage);
                    step();
                }
            }
            ++unit;
            next_unit(count);
        }
    } else if (warp >= 4) {
        // ================================ softmax: a thread per row ================================
        const int x = (warp - 4) >> 2, wq = warp & 3;      // row tile, lane quarter of tensor memory
        const int row = wq * 32 + lane;                    // of the row tile
        const uint32_t lanes = (uint32_t)(wq * 32) << 16;
        const uint32_t o_tm = tmem + 256 + x * 128 + lanes;
        uint32_t k = 0, unit = 0;
        bool ok = true;
        const float sc = p.scale_log2;
        // P V of tile kk done.  A barrier may be one phase behind what is waited for, not two: with two S buffers the
        // softmax can finish a tile while the product before the last still runs, so each buffer has its own.
        auto wait_pv = [&](uint32_t kk) {
            const bool r = NT == 2 ? mbar_wait(pv_done(x), kk & 1u, abort_flag, ws) : mbar_wait(pv_done(kk & 1u), (kk >> 1) & 1u, abort_flag, ws);
            return __all_sync(0xffffffffu, r) != 0;
        };
        while (ok && at < piece_end) {
            const int begin = cur.i, count = (int)min((long long)(cur.t.tiles - cur.i), piece_end - at);
            const Tile t = cur.t;
            const int rows = min(128, t.rows - x * 128);   // of this row tile (can be negative)
            // ---- queries -> shared memory (the S products of the unit before are done: its last S has been read)
            for (int i = row; i < 128 * 8 * DB; i += 128) {
                const int r = i / (8 * DB), ch = i - r * (8 * DB);
                uint4 q = make_uint4(0, 0, 0, 0);
                if (r < rows && ch * 8 < p.D) {
                    const int rr = t.r0 + x * 128 + r, tok = rr / p.g, hg = rr - tok * p.g;
                    q = __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const __nv_bfloat16 *>(p.q) + (int64_t)(cur.start + tok) * p.q_stride +
                                                              (int64_t)(cur.h * p.g + hg) * p.D) + ch);
                }
                const uint32_t a = sq + x * G::kTileBytes + (ch >> 3) * (128 * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(q_ready(x));
            // ---- what the row sees; what all rows of the row tile see
            const bool live = row < rows, warp_live = wq * 32 < rows;
            int hi_r = 0, lo_r = 0, sink_r = 0;
            if (live) {
                const int pos = cur.pre + (t.r0 + x * 128 + row) / p.g;
                hi_r = p.mask == MRP_ATTN_CAUSAL ? pos + 1 : t.hi;
                lo_r = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
                sink_r = p.sinks;
            }
            int all_hi = 0, all_lo = 0;
            if (warp_live) {
                const int a = t.r0 + x * 128 + wq * 32, b = t.r0 + x * 128 + min(rows, wq * 32 + 32) - 1;
                all_hi = p.mask == MRP_ATTN_CAUSAL ? cur.pre + a / p.g + 1 : t.hi;
                all_lo = p.window > 0 ? max(0, cur.pre + b / p.g + 1 - p.window) : 0;
            }
            float m = -INFINITY, l = 0.f;
            for (int n = 0; n < count; ++n, ++k) {
                const int buf = NT == 2 ? x : (int)(k & 1u);
                const uint32_t s_tm = tmem + buf * 128 + lanes;
                ok = __all_sync(0xffffffffu, mbar_wait(s_full(buf), NT == 2 ? k & 1u : (k >> 1) & 1u, abort_flag, ws));
                if (!ok) break;
                tc_fence_after();
                if (warp_live) {
                    float s[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(s_tm + 32 * c, s + 32 * c);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_landed32(s + 32 * c);
                    const int j0 = key_tile(t, begin + n) * kTcTile;
                    if (!(j0 >= all_lo && j0 + kTcTile <= all_hi)) {
#pragma unroll
                        for (int i = 0; i < 128; ++i) {
                            const int j = j0 + i;
                            if (!(j < hi_r && (j >= lo_r || j < sink_r))) s[i] = p.unseen;
                        }
                    }
                    float t0, t1, t2, t3;
                    if (sc > 0.f) {
                        t0 = s[0]; t1 = s[1]; t2 = s[2]; t3 = s[3];
#pragma unroll
                        for (int i = 4; i < 128; i += 4) {
                            t0 = fmaxf(t0, s[i]); t1 = fmaxf(t1, s[i + 1]); t2 = fmaxf(t2, s[i + 2]); t3 = fmaxf(t3, s[i + 3]);
                        }
                        t0 = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3));
                    } else {
                        t0 = s[0]; t1 = s[1]; t2 = s[2]; t3 = s[3];
#pragma unroll
                        for (int i = 4; i < 128; i += 4) {
                            t0 = fminf(t0, s[i]); t1 = fminf(t1, s[i + 1]); t2 = fminf(t2, s[i + 2]); t3 = fminf(t3, s[i + 3]);
                        }
                        t0 = fminf(fminf(t0, t1), fminf(t2, t3));
                    }
                    const float top = t0 * sc;
                    const bool grow = top > m + 8.f;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float nm = grow ? top : m;
                        const float c = m == nm ? 1.f : ex2f(m - nm);
                        if (n > 0) {                       // the accumulator of the tiles so far
                            ok = wait_pv(k - 1);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int f = 0; f < DB * 2; ++f) {
                                float o[32];
                                tmem_ld32(o_tm + 32 * f, o);
                                tmem_wait_ld();
                                tmem_landed32(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] *= c;
                                tmem_st32(o_tm + 32 * f, o);
                            }
                        }
                        l *= c;
                        m = nm;
                    }
                    const float mm = m == -INFINITY ? 0.f : m;
                    float l0 = 0.f, l1 = 0.f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t w[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float a = ex2f(fmaf(s[32 * c + 2 * i], sc, -mm)), b = ex2f(fmaf(s[32 * c + 2 * i + 1], sc, -mm));
                            l0 += a;
                            l1 += b;
                            w[i] = pack_bf16(a, b);
                        }
                        tmem_st16(s_tm + 16 * c, w);
                    }
                    l += l0 + l1;
                    tmem_wait_st();
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(p_ready(buf));
            }
            if (!ok) break;
            // ---- the unit's end (or this piece's)
            ok = wait_pv(k - 1);
            if (!ok) break;
            tc_fence_after();
            if (warp_live) {
                const Suspects &sus = suspects[unit & 1];
                if (sus.n > 0) {
                    bool hit = sus.n > kMaxSuspects;
                    for (int y = 0; y < min(sus.n, kMaxSuspects); ++y)
                        for (int w = 0; w < 4; ++w)
                            for (uint32_t bits = sus.keys[y][w]; bits; bits &= bits - 1) {
                                const int j = sus.base[y] + w * 32 + __ffs(bits) - 1;
                                hit |= j < hi_r && (j >= lo_r || j < sink_r);
                            }
                    if (hit) l = __int_as_float(0x7FC00000);
                }
                const bool whole_unit = count == t.tiles;
                const int rr = t.r0 + x * 128 + row, tok = rr / p.g, head = cur.h * p.g + rr - tok * p.g;
                __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + (int64_t)(cur.start + tok) * p.out_stride + (int64_t)head * p.D;
                float *lse = p.lse ? p.lse + (int64_t)(cur.start + tok) * p.H + head : nullptr;
                auto put = [&](int f0, const float *o, float inv) {        // 8 features from f0
                    if (live && f0 < p.D)
                        *reinterpret_cast<uint4 *>(dst + f0) = make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv),
                                                                          pack_bf16(o[4] * inv, o[5] * inv), pack_bf16(o[6] * inv, o[7] * inv));
                };
                auto inverse = [](float L) { return L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L); };       // (NaN goes through)
                auto put_lse = [&](float M, float L) { if (live && lse) *lse = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f; };
                const int slot = (2 * (int)blockIdx.x + (begin == 0 ? 1 : 0)) * NT + x;
                float4 *part = reinterpret_cast<float4 *>(p.part.o);       // slot: [DB * 16][128 rows] float4
                const float inv = inverse(l);
#pragma unroll
                for (int f = 0; f < DB * 2; ++f) {
                    float o[32];
                    tmem_ld32(o_tm + 32 * f, o);
                    tmem_wait_ld();
                    tmem_landed32(o);
                    if (whole_unit) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8) put(32 * f + i, o + i, inv);
                    } else if (live) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            __stcg(part + ((size_t)slot * (DB * 16) + f * 8 + i) * 128 + row, make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]));
                    }
                }
                if (whole_unit) {
                    put_lse(m, l);
                } else {
                    if (live) __stcg(p.part.ml + (size_t)slot * 128 + row, make_float2(m, l));
                    const int c0 = (int)(cur.unit / per), c1 = (int)((cur.unit + t.tiles - 1) / per);
                    int *counter = p.part.counters + (c0 * NT + x) * 4 + wq;
                    __threadfence();
                    __syncwarp();
                    int last = 0;
                    if (lane == 0) last = atomicAdd(counter, 1) == c1 - c0;
                    last = __shfl_sync(0xffffffffu, last, 0);
                    if (last) {
                        __threadfence();
                        auto slot_of = [&](int c) { return (size_t)((2 * c + (c == c0)) * NT + x); };
                        float M = -INFINITY, L = 0.f;
                        if (live) {
                            for (int c = c0; c <= c1; ++c) M = fmaxf(M, __ldcg(p.part.ml + slot_of(c) * 128 + row).x);
                            for (int c = c0; c <= c1; ++c) {
                                const float2 ml = __ldcg(p.part.ml + slot_of(c) * 128 + row);
                                if (ml.x == -INFINITY && ml.y == 0.f) continue;
                                L = fmaf(ml.x == -INFINITY ? 0.f : ex2f(ml.x - M), ml.y, L);
                            }
                            const float iv = inverse(L);
#pragma unroll 1
                            for (int f = 0; f < DB * 8 && f * 8 < p.D; ++f) {
                                float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                                for (int c = c0; c <= c1; ++c) {
                                    const float2 ml = __ldcg(p.part.ml + slot_of(c) * 128 + row);
                                    const float4 a = __ldcg(part + (slot_of(c) * (DB * 16) + 2 * f) * 128 + row);
                                    const float4 b = __ldcg(part + (slot_of(c) * (DB * 16) + 2 * f + 1) * 128 + row);
                                    const float w = ml.x == -INFINITY ? 0.f : ex2f(ml.x - M);
                                    if (ml.x == -INFINITY && ml.y == 0.f) continue;
                                    o[0] = fmaf(w, a.x, o[0]); o[1] = fmaf(w, a.y, o[1]); o[2] = fmaf(w, a.z, o[2]); o[3] = fmaf(w, a.w, o[3]);
                                    o[4] = fmaf(w, b.x, o[4]); o[5] = fmaf(w, b.y, o[5]); o[6] = fmaf(w, b.z, o[6]); o[7] = fmaf(w, b.w, o[7]);
                                }
                                put(8 * f, o, iv);
                            }
                            put_lse(M, L);
                        }
                        if (lane == 0) *counter = 0;
                    }
                }
                tc_fence_before();
            }
            ++unit;
            next_unit(count);
        }
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

template <int DB, int NT>
cudaError_t tc_prepare()
{
    return cudaFuncSetAttribute(kv_attention_tc_kernel<DB, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcGeo<DB, NT>::kSmem);
}
template <int DB, int NT>
cudaError_t tc_launch(Ctx *c, const AttnParams &p, const CUtensorMap &km, const CUtensorMap &vm, int box, cudaStream_t st)
{
    const int sms = c->sm_count < kKvMaxSm ? c->sm_count : kKvMaxSm;
    cudaError_t e = launch_k(kv_attention_tc_kernel<DB, NT>, dim3(sms), dim3(TcGeo<DB, NT>::kThreads), TcGeo<DB, NT>::kSmem, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p, km, vm, box);
    c->launches = 1;
    return note_err(c, e, "kv_attention_tc_kernel");
}

// Rows of a TMA box: pages of 8, 16, 32 or 64 rows whole, larger ones in 128-row parts; 0: other sizes.
int tc_box_rows(int page_size)
{
    if (page_size % kTcTile == 0) return kTcTile;
    for (int r = 8; r < kTcTile; r *= 2)
        if (page_size == r) return r;
    return 0;
}

bool page_map(Ctx *c, CUtensorMap *map, const void *pool, int box)
{
    const mrp_kv_config &kv = c->kv;
    const cuuint64_t dims[4] = {(cuuint64_t)kv.head_dim, (cuuint64_t)kv.page_size, (cuuint64_t)kv.n_kv_heads, (cuuint64_t)kv.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)kv.head_dim * 2, (cuuint64_t)kv.page_size * kv.head_dim * 2, (cuuint64_t)kv.page_stride * 2};
    const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, es[4] = {1, 1, 1, 1};
    return ((EncodeTiledFn)c->kv_encode)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(pool), dims, strides, boxes, es,
                                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool kv_tc_takes(const mrp_config &cfg, const mrp_kv_config &kv)
{
    // (strides of a tensor map: multiples of 16 bytes below 2^40; heads narrower than 64 would be mostly padding)
    return cfg.dtype == MRP_BF16 && kv.n_pages > 0 && kv.head_dim >= 64 && kv.head_dim <= 128 && tc_box_rows(kv.page_size) > 0 &&
           kv.page_stride < (1ll << 39) && (long long)kv.page_size * kv.head_dim < (1ll << 39) && !(cfg.flags & MRP_FLAG_FORCE_SIMT);
}

size_t kv_tc_workspace_bytes()
{
    return kKvCounterBytes + (size_t)2 * kKvMaxSm * 2 * 128 * (128 * 4 + 8);
}

cudaError_t kv_tc_attach(Ctx *c)
{
    c->kv_encode = nullptr;
    if (!kv_tc_takes(c->cfg, c->kv)) return cudaSuccess;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
    if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) return e != cudaSuccess ? e : cudaErrorNotSupported;
    if ((e = tc_prepare<1, 1>()) != cudaSuccess || (e = tc_prepare<1, 2>()) != cudaSuccess || (e = tc_prepare<2, 1>()) != cudaSuccess ||
        (e = tc_prepare<2, 2>()) != cudaSuccess)
        return e;
    c->kv_encode = fn;
    return cudaSuccess;
}

cudaError_t launch_paged_attention_tc(Ctx *c, AttnParams &p, int max_new, cudaStream_t st)
{
    const int box = tc_box_rows(c->kv.page_size);
    CUtensorMap km, vm;
    if (!page_map(c, &km, p.k, box) || !page_map(c, &vm, p.v, box)) return note_err(c, cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
    const size_t slots = (size_t)2 * kKvMaxSm * 2;
    p.part.counters = (int32_t *)c->kv_ws;
    p.part.ml = (float2 *)(c->kv_ws + kKvCounterBytes);
    p.part.o = (float *)(c->kv_ws + kKvCounterBytes + slots * 128 * 8);
    const bool two = (long long)max_new * p.g > 128;
    if (c->kv.head_dim <= 64) return two ? tc_launch<1, 2>(c, p, km, vm, box, st) : tc_launch<1, 1>(c, p, km, vm, box, st);
    return two ? tc_launch<2, 2>(c, p, km, vm, box, st) : tc_launch<2, 1>(c, p, km, vm, box, st);
}

}  // namespace mrp

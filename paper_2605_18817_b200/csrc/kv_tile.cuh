// What the attention kernels on large tiles share (kv_attention_tc.cu, kv_attention_q8.cu): tiles of 128 keys in 128-byte-swizzled
// stages, how they are fetched, cleaned and (8 bits) turned into bf16, tensor-memory access, the joining of pieces.
#pragma once
#include <cuda_fp16.h>

#include "kv_attention.cuh"
#include "kv_q8.cuh"
#include "tc_common.cuh"

namespace mrp {
namespace {

constexpr int kTcTile = 128;               // keys of a tile, rows of a row tile
constexpr int kMaxSuspects = 16;           // boundary tiles of a unit that are remembered for values that are not finite

struct WaitStatus {
    int32_t *status, *user_status;
};

// A head is NB blocks of 64 features (1, 2 or 4); a ring stage holds DB of them (1 or 2) of a K or V tile, HB stages a tile.
template <int NB> struct Blocks {
    static constexpr int DB = NB >= 2 ? 2 : 1, HB = NB / DB;
    static constexpr int kStageBytes = DB * 128 * 128;
};
// How the keys and values lie (see TileAt, PageBoxes): pages, a box a 64-feature block (kApart) or two (kJoined); rows beside the
// queries (kPacked); pages of 8 bits (kCodes).
enum { kApart = 0, kJoined = 1, kPacked = 2, kCodes = 3 };

// What a role's loop does rarely stands outside of it: the loops of all roles have to stay in the instruction caches together.
__device__ __noinline__ bool wait_longer(uint32_t bar, uint32_t parity, volatile int *abort_flag, int32_t *status, int32_t *user_status)
{
    const WaitStatus ws = {status, user_status};
    return mbar_wait(bar, parity, abort_flag, ws);
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, const WaitStatus &ws)
{
    return mbar_try_wait(bar, parity) || wait_longer(bar, parity, abort_flag, ws.status, ws.user_status);
}
template <int ROWS>
__device__ __noinline__ void next_unit(const AttnParams &p, Cursor<ROWS, kTcTile> &c, int places, long long piece_end) { leave_unit(p, c, places, piece_end); }

// find_piece for a warp on its own, of any number of sequences, in little code (twice through them).
template <int ROWS>
__device__ __noinline__ long long cut_line(const AttnParams &p, Cursor<ROWS, kTcTile> &c, long long &per, bool report)
{
    const int lane = threadIdx.x & 31;
    long long begin = 0, end = 0, done = 0, mine = 0;
    c.s = -1;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
        for (int s0 = 0; s0 < p.b.n_seqs && c.s < 0; s0 += 32) {
            if (pass == 0 || p.b.n_seqs > 32) mine = s0 + lane < p.b.n_seqs ? sequence_tiles<ROWS, kTcTile>(p, s0 + lane, pass == 0 && report) : 0;
            long long x = mine;
            if (pass == 0) {
#pragma unroll
                for (int w = 16; w > 0; w >>= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
                done += x;
                continue;
            }
#pragma unroll
            for (int w = 1; w < 32; w <<= 1) {             // inclusive sum over the lanes
                const long long y = __shfl_up_sync(0xffffffffu, x, w);
                if (lane >= w) x += y;
            }
            const long long before = done + x - mine;
            const uint32_t hit = __ballot_sync(0xffffffffu, mine > 0 && before <= begin && begin < before + mine);
            if (hit) {
                c.s = s0 + __ffs(hit) - 1;
                c.at = __shfl_sync(0xffffffffu, before, __ffs(hit) - 1);
            }
            done += __shfl_sync(0xffffffffu, x, 31);
        }
        if (pass == 0) {
            per = div_line(done + gridDim.x - 1, gridDim.x);
            begin = per * blockIdx.x;
            end = min(done, begin + per);
            if (begin >= end) return 0;
            done = 0;
        }
    }
    kv_sequence(p.b, c.s, c.start, c.n, c.pre);
    c.rt = -1;
    long long next = c.at;
    do {                                   // the row tile
        c.at = next;
        c.t = row_tile<ROWS, kTcTile>(p, c.n, c.pre, ++c.rt);
        next = c.at + (long long)(c.t.tiles + p.lead) * p.Hk;
    } while (next <= begin);
    const int in = (int)(begin - c.at);
    c.h = in / (c.t.tiles + p.lead);
    c.i = in - c.h * (c.t.tiles + p.lead);
    c.at = begin;
    c.unit = begin - c.i;
    return end - begin;
}

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
__device__ __forceinline__ void tmem_ld16_go(uint32_t a, float *v)         // 16 columns; no wait
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_landed16(float *v)
{
    asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                      "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]) :: "memory");
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

constexpr int kFewRows = 16;
constexpr float kNone = -3.4028234e38f;    // the maximum of a row that has seen nothing

template <int N> __device__ __forceinline__ void tmem_ld_n(uint32_t a, float *v);
template <> __device__ __forceinline__ void tmem_ld_n<32>(uint32_t a, float *v)
{
    tmem_ld32(a, v);
    tmem_wait_ld();
    tmem_landed32(v);
}
template <> __device__ __forceinline__ void tmem_ld_n<16>(uint32_t a, float *v)
{
    tmem_ld16_go(a, v);
    tmem_wait_ld();
    tmem_landed16(v);
}
__device__ __forceinline__ void wg_sync(int id) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool any_of(int id, int threads, bool x)        // barrier of `threads` threads, true where any one's x is
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbarrier.cta.red.or.pred q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(id), "r"(threads), "r"((uint32_t)x) : "memory");
    return r != 0;
}
__device__ __forceinline__ bool wg_any(int id, bool x) { return any_of(id, 128, x); }
// Reduces W rows (a value per lane each) over the warp; lane i returns row i (i % W).  Each step halves the rows a lane goes
// on with: W - 1 exchanges instead of 5 W.
template <int W, bool MAX> __device__ __forceinline__ float reduce_rows(float (&s)[W], int lane)
{
    auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
#pragma unroll
    for (int h = W / 2; h > 0; h >>= 1) {
        const bool up = (lane & h) != 0;
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float keep = up ? s[i + h] : s[i], send = up ? s[i] : s[i + h];
            s[i] = op(keep, __shfl_xor_sync(0xffffffffu, send, h));
        }
    }
    float r = s[0];
#pragma unroll
    for (int h = W; h < 32; h <<= 1) r = op(r, __shfl_xor_sync(0xffffffffu, r, h));
    return r;
}

// Two fp32 operations in one instruction: (a, b) * s + c, (a, b) + (c, d)
__device__ __forceinline__ void fma2(float &a, float &b, float s, float c)
{
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(s), "f"(c));
}
__device__ __forceinline__ void add2(float &a, float &b, float c, float d)
{
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
// bits lo..hi-1 of 32
__device__ __forceinline__ uint32_t bit_range(int lo, int hi)
{
    const uint32_t h = hi >= 32 ? ~0u : hi <= 0 ? 0u : (1u << hi) - 1u, l = lo >= 32 ? ~0u : lo <= 0 ? 0u : (1u << lo) - 1u;
    return h & ~l;
}

// K as an operand whose contraction runs along its rows (features), groups of 8 rows `group` bytes apart
__device__ __forceinline__ uint64_t k_desc(uint32_t saddr, uint32_t group)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)1 << 16;
    d |= (uint64_t)(group >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// V^T as the A operand, V or P as the B operand: rows (keys) of 128 bytes, MN-major; `block` bytes to the next 64 features,
// `group` to the next 8 keys
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr, uint32_t block, uint32_t group)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(block >> 4) << 16;
    d |= (uint64_t)(group >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// How pages become tiles.  A box is `rows` rows of one page and key head: 64 features wide, a box per 64-feature block, the
// blocks of a tile 16 KB apart; or JOINED, where a page holds whole blocks of 128 features: 128 features wide (the pool seen
// as [groups of 8 rows][64-feature block][row of the group][64 features]), the two blocks of a group of 8 rows side by side.
// Half as many boxes of twice the size: with small pages their number is what bounds the stream.
struct PageBoxes {
    int rows;
    int page_groups, head_groups, groups;  // joined (else 0): groups of 8 rows from page to page, head to head, in all
};
template <int DB, int LAY> struct TileAt {                 // of a tile: bytes to the next 64-feature block, the next group of 8 keys
    static constexpr uint32_t block = LAY == kJoined ? 1024 : 128 * 128, group = LAY == kJoined ? DB * 1024 : 1024;
};

// The box of a tile's keys that is the lane's: where it lies in the pool.  Looked up a tile ahead of its use.
struct PageRef {
    bool need;                 // holds visible positions
    int entry, row;            // page, row in it
};
template <int LAY, typename Tile>
__device__ __forceinline__ PageRef look_up(const AttnParams &p, const PageBoxes &bx, const Tile &t, int n, int s, int start, int lane)
{
    const int j = key_tile(t, n) * kTcTile + lane * bx.rows;
    PageRef r;
    r.need = lane * bx.rows < kTcTile && ((j < t.hi && j + bx.rows > t.lo) || j < t.s1);
    r.entry = r.row = 0;
    if (LAY == kPacked) {
        r.row = start + j;                                 // (rows behind the sequence's: not seen, whatever they are)
    } else if (r.need) {
        const int pg = fast_div(j, p.b.page);
        r.row = j - pg * p.b.page.d;
        r.entry = __ldg(p.b.page_table + (size_t)s * p.b.max_pages + pg);
    }
    return r;
}

// The pages of a K or V tile's visible positions, 64 DB features from `feature` on -> a ring stage; the whole warp.
template <int DB, int LAY>
__device__ __forceinline__ void fetch_tile(const AttnParams &p, const CUtensorMap *map, const PageBoxes &bx, const PageRef &r, int h, int feature,
                                           uint32_t dst, uint32_t bar, int lane)
{
    const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, r.need));
    if (lane == 0) mbar_expect_tx(bar, boxes * bx.rows * 128u * DB);
    __syncwarp();
    if (r.need) {
        const bool bad = LAY != kPacked && (unsigned)r.entry >= (unsigned)p.b.n_pages;
        if (bad) kv_bad_index(p.b);
        dst += lane * (bx.rows >> 3) * TileAt<DB, LAY>::group;
        // (a page that is not one: outside the map, zeros arrive)
        if (LAY == kJoined) {
            const int g = bad ? bx.groups : r.entry * bx.page_groups + h * bx.head_groups + (r.row >> 3);
            tma_load_page(dst, map, 0, 0, feature >> 6, g, bar);
        } else {
#pragma unroll
            for (int x = 0; x < DB; ++x)
                tma_load_page(dst + x * (128 * 128), map, feature + 64 * x, r.row, h, bad ? p.b.n_pages : r.entry, bar);
        }
    }
}

// 8 bits: the same, 128 keys of `pitch` codes from `feature` on, one row after the other, -> a raw stage.
__device__ __forceinline__ void fetch_codes(const AttnParams &p, const CUtensorMap *map, const PageBoxes &bx, const PageRef &r, int h, int feature,
                                            int pitch, uint32_t dst, uint32_t bar, int lane)
{
    const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, r.need));
    if (lane == 0) mbar_expect_tx(bar, boxes * bx.rows * (uint32_t)pitch);
    __syncwarp();
    if (r.need) {
        const bool bad = (unsigned)r.entry >= (unsigned)p.b.n_pages;
        if (bad) kv_bad_index(p.b);
        tma_load_page(dst + lane * bx.rows * pitch, map, feature, r.row, h, bad ? p.b.n_pages : r.entry, bar);
    }
}

// Codes -> bf16: a code's bits, moved to a bf16's sign, lower exponent and upper mantissa bits, are its value times 2^-120 (subnormal
// codes: subnormal bf16), so one exact product with 2^(s - 7) is all there is to a row of scale byte s; scales above 2^7 take two.
struct Turn {
    uint32_t f, g;             // bf16 twice
};
__device__ __forceinline__ Turn turn_of(uint32_t s, bool seen)             // a key's factors; 0 where no row sees it
{
    const uint32_t a = !seen ? 0u : s == kQ8NaN ? 0x7FC0u : (min(s, 134u) + 120u) << 7, b = s > 134u && s != kQ8NaN ? (s - 7u) << 7 : 0x3F80u;
    return Turn{a | a << 16, b | b << 16};
}
__device__ __forceinline__ uint32_t times_bf16(uint32_t x, uint32_t f)
{
    const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&f));
    return *reinterpret_cast<const uint32_t *>(&y);
}
template <uint32_t SEL> __device__ __forceinline__ uint32_t prmt(uint32_t x)   // (with the selector's sign bits, which __byte_perm drops)
{
    uint32_t y;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(y) : "r"(x), "n"(SEL));
    return y;
}
// 4 codes -> 2 x 2 bf16.  (Each byte beside its sign, 8 times, then moved up: the sign lands on bit 15, the others on 4 to 10.)
__device__ __forceinline__ void turn_four(uint32_t x, uint32_t f, uint32_t &lo, uint32_t &hi)
{
    lo = times_bf16((prmt<0x9180>(x) << 4) & 0x87F087F0u, f);
    hi = times_bf16((prmt<0xB3A2>(x) << 4) & 0x87F087F0u, f);
}

// The scale bytes of a warp's keys of a tile (32 KR of them from `first` on, lane l: keys l, l + 32, ..), in two steps: the pages they
// lie in, the bytes.
template <int KR> struct KeyPlaces {
    int entry[KR], row[KR];    // entry -1: no row sees the key
};
template <int KR, typename Tile>
__device__ __forceinline__ KeyPlaces<KR> find_keys(const AttnParams &p, const Tile &t, bool there, int i, int s, int first, int lane)
{
    KeyPlaces<KR> a;
#pragma unroll
    for (int y = 0; y < KR; ++y) {
        const int j = there ? key_tile(t, i) * kTcTile + first + y * 32 + lane : t.hi;
        a.entry[y] = -1;
        a.row[y] = 0;
        if (j < t.hi && (j >= t.lo || j < t.s1)) {
            const int pg = fast_div(j, p.b.page);
            a.row[y] = j - pg * p.b.page.d;
            a.entry[y] = __ldg(p.b.page_table + (size_t)s * p.b.max_pages + pg);
        }
    }
    return a;
}
// 256: no row sees the key, or its page is none
template <int KR>
__device__ __forceinline__ void load_scales(const AttnParams &p, const uint8_t *scale, const KeyPlaces<KR> &a, int h, uint32_t (&s)[KR])
{
#pragma unroll
    for (int y = 0; y < KR; ++y) {
        s[y] = 256u;
        if ((unsigned)a.entry[y] < (unsigned)p.b.n_pages) s[y] = __ldg(scale + ((int64_t)a.entry[y] * p.Hk + h) * p.b.page.d + a.row[y]);
    }
}

// A raw stage (128 keys of `pitch` codes) -> a stage of the ring, 64 DB features (those from `wide` on: zeros): a warp's 32 KR keys
// from key0 on, with their scale bytes.  Four lanes a key, 16 codes each at a time; of two feature blocks neighbouring keys take
// different ones, so that loads and (swizzled) stores touch every bank once.
template <int DB, int KR>
__device__ __forceinline__ void turn_stage(uint32_t from, uint32_t to, int key0, int pitch, int wide, const uint32_t (&bytes)[KR], int lane)
{
    constexpr int N = 4 * KR;                              // rounds of 8 keys
    const int kk = lane >> 2, q = lane & 3;
    Turn own[KR];
    bool any = false;
#pragma unroll
    for (int y = 0; y < KR; ++y) {
        own[y] = turn_of(bytes[y], bytes[y] < 256u);
        any |= own[y].g != 0x3F803F80u && bytes[y] < 256u;
    }
    const bool large = __any_sync(0xffffffffu, any);
    uint32_t load_at[DB], store_at[DB];
    bool in[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const int ch = q + (DB == 2 ? 4 * (d ^ (kk & 1)) : 0);
        in[d] = ch * 16 < wide;
        load_at[d] = from + (key0 + kk) * pitch + (in[d] ? ch * 16 : 0);       // (beyond: any codes, times zero)
        store_at[d] = to + (key0 >> 3) * 1024 + kk * 128 + (ch >> 2) * (128 * 128);
    }
    const uint32_t s0 = ((2 * q) ^ kk) << 4, s1 = ((2 * q + 1) ^ kk) << 4;
    // (a short loop: the roles of a kernel share the instruction caches.  Unrolled it took twice as long)
#pragma unroll 1
    for (int r = 0; r < N; r += 2) {
        uint32_t c[2][DB][4], f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 0; d < DB; ++d)
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(c[e][d][0]), "=r"(c[e][d][1]), "=r"(c[e][d][2]), "=r"(c[e][d][3])
                             : "r"(load_at[d] + (r + e) * 8 * pitch) : "memory");
        const uint32_t fo = KR == 2 && r >= 4 ? own[KR - 1].f : own[0].f;
#pragma unroll
        for (int e = 0; e < 2; ++e) f[e] = __shfl_sync(0xffffffffu, fo, ((r + e) & 3) * 8 + kk);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const uint32_t fd = in[d] ? f[e] : 0u, at = store_at[d] + (r + e) * 1024;
                uint32_t o[8];
#pragma unroll
                for (int z = 0; z < 4; ++z) turn_four(c[e][d][z], fd, o[2 * z], o[2 * z + 1]);
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at + s0), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at + s1), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
            }
    }
    if (large) {                                           // the second factor, over what this lane has stored
#pragma unroll 1
        for (int r = 0; r < N; ++r) {
            uint32_t g = r < 4 ? own[0].g : own[KR - 1].g;
            g = __shfl_sync(0xffffffffu, g, (r & 3) * 8 + kk);
#pragma unroll 1
            for (int d = 0; d < 2 * DB; ++d) {
                const uint32_t at = store_at[DB == 2 ? d >> 1 : 0] + r * 1024 + (d & 1 ? s1 : s0);
                uint32_t o[4];
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]) : "r"(at) : "memory");
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(times_bf16(o[0], g)), "r"(times_bf16(o[1], g)), "r"(times_bf16(o[2], g)),
                             "r"(times_bf16(o[3], g)) : "memory");
            }
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

// Query rows r0.. of a tile (those below `rows`; zeros beyond, and beyond the head's features) -> shared memory, as K-major
// blocks of 64 features.  THREADS threads, all copies in flight together.
template <int NB, int ROWS, int THREADS>
__device__ __forceinline__ void load_queries(const AttnParams &p, int start, int h, int r0, int rows, uint32_t sq, int tid)
{
    constexpr int kRow = 8 * NB, kStep = THREADS / kRow;   // 16-byte chunks of a row; rows a round
    static_assert(THREADS % kRow == 0 && ROWS % kStep == 0, "whole rounds");
    const int ch = tid % kRow;
    const __nv_bfloat16 *src = reinterpret_cast<const __nv_bfloat16 *>(p.q) + (int64_t)start * p.q_stride + (int64_t)h * p.g * p.D;
    const bool wide = ch * 8 < p.D;
    int r = tid / kRow, tok = fast_div(r0 + r, p.gdiv), hg = r0 + r - tok * p.g;
    const int dt = fast_div(kStep, p.gdiv), dh = kStep - dt * p.g;
    uint32_t a = sq + (ch >> 3) * (ROWS * 128) + r * 128;
#pragma unroll 4
    for (int i = 0; i < ROWS / kStep; ++i) {
        const bool on = wide & (r < rows);
        const __nv_bfloat16 *q = on ? src + (int64_t)tok * p.q_stride + hg * p.D + ch * 8 : src;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(a + (((ch & 7) ^ (r & 7)) << 4)), "l"(q), "r"(on ? 16 : 0) : "memory");
        r += kStep;
        a += kStep * 128;
        tok += dt;
        hg += dh;
        if (hg >= p.g) { hg -= p.g; ++tok; }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// What a unit's rows see together, for the V rows that must not reach a product: rows no row sees -> zeros; rows some
// see that hold what is not finite -> zeros, remembered.  One warp, on a V tile that has landed.
struct Seen {
    int all_lo, all_hi;
    bool differ;
};
template <typename Tile>
__device__ __forceinline__ Seen seen_by_all(const AttnParams &p, const Tile &t, int pre)
{
    const int i0 = fast_div(t.r0, p.gdiv), i1 = fast_div(t.r0 + t.rows - 1, p.gdiv);
    Seen s;
    s.differ = i0 != i1 && (p.mask == MRP_ATTN_CAUSAL || p.window > 0);
    s.all_hi = p.mask == MRP_ATTN_CAUSAL ? pre + i0 + 1 : t.hi;
    s.all_lo = p.window > 0 ? max(0, pre + i1 + 1 - p.window) : 0;
    return s;
}
template <int DB, int LAY, typename Tile>
__device__ __forceinline__ void clean_tile(const Tile &t, const Seen &a, int j0, uint32_t vs, Suspects &sus, int lane)
{
    typedef TileAt<DB, LAY> lay;
    if ((j0 >= t.lo && j0 + kTcTile <= t.hi) || j0 + kTcTile <= t.s1) {
        if (!a.differ || (j0 >= a.all_lo && j0 + kTcTile <= a.all_hi)) return;
    }
    uint32_t found[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int row = w * 32 + lane, j = j0 + row;
        const uint32_t at = vs + (row >> 3) * lay::group + (row & 7) * 128;
        const bool seen = j < t.hi && (j >= t.lo || j < t.s1);
        bool bad = false;
        if (seen && a.differ && !(j >= a.all_lo && j < a.all_hi)) {
            for (int c = 0; c < 8 * DB; ++c) {
                uint32_t u[4];
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                             : "r"(at + (c >> 3) * lay::block + (((c + lane) & 7) << 4)) : "memory");
#pragma unroll
                for (int y = 0; y < 4; ++y) bad |= (u[y] & 0x7F800000u) == 0x7F800000u || (u[y] & 0x7F80u) == 0x7F80u;
            }
        }
        found[w] = __ballot_sync(0xffffffffu, bad);
        if (!seen || bad)
            for (int c = 0; c < 8 * DB; ++c)
                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};"
                             ::"r"(at + (c >> 3) * lay::block + (((c + lane) & 7) << 4)), "r"(0u) : "memory");
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
}
// The same as a short function, for apart tiles.
template <int DB, typename Tile>
__device__ __noinline__ void clean_rarely(const Tile &t, const Seen &a, int j0, uint32_t vs, Suspects &sus, int lane)
{
    typedef TileAt<DB, kApart> lay;
    if (((j0 >= t.lo && j0 + kTcTile <= t.hi) || j0 + kTcTile <= t.s1) && (!a.differ || (j0 >= a.all_lo && j0 + kTcTile <= a.all_hi))) return;
    int slot = -1;
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
        const int row = w * 32 + lane, j = j0 + row;
        const uint32_t at = vs + (row >> 3) * lay::group + (row & 7) * 128;
        const bool seen = j < t.hi && (j >= t.lo || j < t.s1);
        bool bad = false;
        if (seen && a.differ && !(j >= a.all_lo && j < a.all_hi)) {
#pragma unroll 2
            for (int c = 0; c < 8 * DB; ++c) {
                uint32_t u[4];
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                             : "r"(at + (c >> 3) * lay::block + (((c + lane) & 7) << 4)) : "memory");
#pragma unroll
                for (int y = 0; y < 4; ++y) bad |= (u[y] & 0x7F800000u) == 0x7F800000u || (u[y] & 0x7F80u) == 0x7F80u;
            }
        }
        const uint32_t found = __ballot_sync(0xffffffffu, bad);
        if (!seen || bad)
#pragma unroll 2
            for (int c = 0; c < 8 * DB; ++c)
                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at + (c >> 3) * lay::block + (((c + lane) & 7) << 4)), "r"(0u) : "memory");
        if (found) {
            if (slot < 0) {
                slot = sus.n;
                __syncwarp();
                if (lane == 0) {
                    if (slot < kMaxSuspects) {
                        sus.base[slot] = j0;
                        sus.keys[slot][0] = sus.keys[slot][1] = sus.keys[slot][2] = sus.keys[slot][3] = 0;
                    }
                    sus.n = slot + 1;
                }
            }
            if (lane == 0 && slot < kMaxSuspects) sus.keys[slot][w] = found;
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}
__device__ __forceinline__ bool suspects_hit(const Suspects &sus, int hi, int lo, int sinks)
{
    bool hit = sus.n > kMaxSuspects;
    for (int y = 0; y < min(sus.n, kMaxSuspects); ++y)
        for (int w = 0; w < 4; ++w)
            for (uint32_t bits = sus.keys[y][w]; bits; bits &= bits - 1) {
                const int j = sus.base[y] + w * 32 + __ffs(bits) - 1;
                hit |= sees(j, hi, lo, sinks);
            }
    return hit;
}

__device__ __forceinline__ float inverse(float l) { return l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l); }      // (NaN goes through)
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f; }

// Joins the pieces c0..c1 of a unit in their order, with a running maximum: warp w of four takes every fourth row, RG rows
// and U pieces of each in flight, a lane four features.
struct JoinArgs {
    const float2 *ml;
    const float *o;
    __nv_bfloat16 *out;                    // of the unit's sequence and key head
    float *lse;
    int64_t out_stride;
    int H, D, g;
    FastDiv gdiv;
    int r0, rows, c0, c1;
};
__device__ __forceinline__ JoinArgs join_args(const AttnParams &p, int start, int h, int r0, int rows, int c0, int c1)
{
    JoinArgs a;
    a.ml = p.part.ml;
    a.o = p.part.o;
    a.out = reinterpret_cast<__nv_bfloat16 *>(p.out) + (int64_t)start * p.out_stride + (int64_t)h * p.g * p.D;
    a.lse = p.lse ? p.lse + (int64_t)start * p.H + h * p.g : nullptr;
    a.out_stride = p.out_stride;
    a.H = p.H; a.D = p.D; a.g = p.g; a.gdiv = p.gdiv;
    a.r0 = r0; a.rows = rows; a.c0 = c0; a.c1 = c1;
    return a;
}
template <int NR, int WIDE, int RG, int U>
__device__ __forceinline__ void join_rows(const JoinArgs &p, int w, int lane)
{
    const int rows = p.rows, c0 = p.c0, c1 = p.c1;
#pragma unroll 1
    for (int f0 = 0; f0 < WIDE; f0 += 128) {
        const bool mine = f0 + 4 * lane < p.D;
#pragma unroll 1
        for (int rb = w; rb < rows; rb += 4 * RG) {
            float M[RG], L[RG];
            float4 a[RG];
#pragma unroll
            for (int y = 0; y < RG; ++y) { M[y] = kNone; L[y] = 0.f; a[y] = make_float4(0.f, 0.f, 0.f, 0.f); }
#pragma unroll 1
            for (int cb = c0; cb <= c1; cb += U) {
                float2 ml[RG][U];
                float4 o[RG][U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int c = min(cb + i, c1);
                    const size_t sl = (size_t)(2 * c + (c == c0)) * NR;
#pragma unroll
                    for (int y = 0; y < RG; ++y) {
                        const int r = min(rb + 4 * y, rows - 1);
                        ml[y][i] = __ldcg(p.ml + sl + r);
                        o[y][i] = __ldcg(reinterpret_cast<const float4 *>(p.o + (sl + r) * WIDE) + (mine ? f0 / 4 + lane : 0));
                    }
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (cb + i <= c1) {
#pragma unroll
                        for (int y = 0; y < RG; ++y) {
                            const float nm = fmaxf(M[y], ml[y][i].x);
                            const float f = M[y] == nm ? 1.f : ex2f(M[y] - nm), e = ml[y][i].x == nm ? 1.f : ex2f(ml[y][i].x - nm);
                            M[y] = nm;
                            L[y] = fmaf(e, ml[y][i].y, L[y] * f);
                            a[y].x = fmaf(e, o[y][i].x, a[y].x * f); a[y].y = fmaf(e, o[y][i].y, a[y].y * f);
                            a[y].z = fmaf(e, o[y][i].z, a[y].z * f); a[y].w = fmaf(e, o[y][i].w, a[y].w * f);
                        }
                    }
            }
#pragma unroll
            for (int y = 0; y < RG; ++y) {
                const int r = rb + 4 * y;
                if (r < rows && mine) {
                    const float inv = inverse(L[y]);
                    const int rr = p.r0 + r, tok = fast_div(rr, p.gdiv), hg = rr - tok * p.g;
                    __nv_bfloat16 *dst = p.out + (int64_t)tok * p.out_stride + (int64_t)hg * p.D + f0 + 4 * lane;
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(a[y].x * inv, a[y].y * inv), pack_bf16(a[y].z * inv, a[y].w * inv));
                    if (f0 + lane == 0 && p.lse) p.lse[(int64_t)tok * p.H + hg] = log_sum(M[y], L[y]);
                }
            }
    }
    }
}

}  // namespace

bool codes_map(Ctx *c, CUtensorMap *map, const void *pool, int box_rows, bool swizzled);       // (kv_attention_q8.cu)

}  // namespace mrp

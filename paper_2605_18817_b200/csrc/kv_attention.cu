// Attention over the pages of a key / value cache: the launch of all forms, and the kernel on warp-level products, which serves
// f32 contexts, pages that are no multiple of 8 rows, and MRP_FLAG_FORCE_SIMT (bf16 otherwise: kv_attention_tc.cu).
//
//   out_r = sum_j p_rj V_j / sum_j p_rj,  p_rj = exp2(scale log2(e) (q_r . K_j) - m_r)  over the visible positions j,
// m_r the running maximum (raised only when a score exceeds it by 2^8, which keeps p and its sum well inside fp32 and
// bf16 and spares most rescalings of the accumulator), p_rj and its sum in fp32.
//
// Decoding reads every K / V row once and does little else.  The g = n_heads / n_kv_heads query heads
// that share a key head and the new tokens of a sequence are the rows of one tile (row r = token r / g, head r % g; 16
// rows), so a K / V row is read once for all of them.  The keys of a (sequence, row tile, key head) unit go in tiles of
// 64, 16 for each of the CTA's four warps; a warp keeps its own ring of 16-key stages filled by cp.async ahead of its
// products and meets the other warps only at the end of a unit.  All tiles of all units form one line that is cut into
// equal pieces, one per CTA of a grid that fills the GPU: ragged batches balance to one tile, and a unit cut in two or
// more pieces is joined by the CTA that finishes last (an arrival counter; nobody waits).  The lengths are read on the
// device, so the cut is found there: every CTA sums the units' tiles itself.
//
// bf16: mma.sync m16n8k16, operands by ldmatrix from XOR-swizzled rows, probabilities as bf16 hi + lo.
// f32:  mma.sync m16n8k8 on tf32 operands split into two (x = hi + lo, three products: relative 2^-21).
//
// What bounds it: the instructions around the products (f32: splitting K and V, three conversions and a subtraction a value and
// row of the tile), not memory.  24 sequences of 200 to 6000 positions, one token each, 32 / 8 heads: bf16 of 128 features in
// pages of 20 rows 100 us (48 for the bytes); f32 107 (48) at 64 features, 184 (97) at 128, 530 (193) at 256.  Two CTAs an SM
// count more than a second stage: f32 of 128 features 235 us with two stages of one CTA.  Rows beyond 16 take a unit per 16.
#include "kv_attention.cuh"

namespace mrp {
namespace {

constexpr int kRows = 16;                  // query rows of a tile
constexpr int kTile = 64;                  // keys of a tile
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kWarpKeys = kTile / kWarps;  // 16
constexpr float kLazy = 8.f;               // log2 of the growth a running maximum may lag behind

__device__ __forceinline__ uint32_t s_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool read)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(read ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t r[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t r[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma16(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma8(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x = hi + lo, both tf32 (10 mantissa bits and a sign each): what is left out is below 2^-21 of x
__device__ __forceinline__ void split_tf32(float x, uint32_t &hi, uint32_t &lo)
{
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(x));
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(lo) : "f"(x - __uint_as_float(hi)));
}
// hi = bf16(a, b); lo = bf16 of what the rounding left out
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &hi, uint32_t &lo)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    hi = *reinterpret_cast<const uint32_t *>(&h);
    const __nv_bfloat162 l = __floats2bfloat162_rn(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xFFFF0000u));
    lo = *reinterpret_cast<const uint32_t *>(&l);
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- element types -------------------------------------------------------------------------------------------------
template <typename T, int DP> struct Geo;
template <int DP> struct Geo<__nv_bfloat16, DP> {
    static constexpr int kChunks = DP / 8;                 // 16-byte chunks of a row
    static constexpr int kPitchK = DP * 2, kPitchV = DP * 2, kPitchQ = DP * 2;     // bytes; chunks XOR-swizzled
    static constexpr int kStages = DP <= 64 ? 3 : 2;
    static constexpr bool kSwizzle = true;
};
template <int DP> struct Geo<float, DP> {
    static constexpr int kChunks = DP / 4;
    static constexpr int kPitchK = DP * 4 + 32, kPitchV = DP * 4 + 16, kPitchQ = DP * 4 + 32;
    static constexpr int kStages = DP <= 64 ? 2 : 1;
    static constexpr bool kSwizzle = false;
};
template <typename T, int DP> struct Smem {
    typedef Geo<T, DP> G;
    static constexpr int kStage = kWarpKeys * (G::kPitchK + G::kPitchV);
    static constexpr int kRing = kWarps * G::kStages * kStage;
    static constexpr int kQ = kRows * G::kPitchQ;
    static constexpr int kRedPitch = DP + 4;               // floats
    static constexpr int kRed = kWarps * kRows * kRedPitch * 4;
    static constexpr int kMl = 2 * kWarps * kRows * 4;
    static constexpr int kTotal = kRing + kQ + kRed + kMl;
    static constexpr int kCtas = kTotal <= 113 * 1024 ? 2 : 1;
};

template <int DP>
__device__ __forceinline__ uint32_t chunk_at(uint32_t base, int row, int chunk)    // bf16 rows
{
    return base + row * (DP * 2) + ((chunk ^ (row & 7)) << 4);
}

// Zeroes values that are not finite in rows that some but not all query rows see, after adding them to the rows that
// do: 0 * inf must not reach the others.  p[nt][4]: the warp's probabilities; v: the warp's 16 value rows.  f32: the numbers that
// round to infinity as tf32 too (from 2^128 - 2^116 on).
template <typename T, int DP, int NF>
__device__ __noinline__ void patch_nonfinite(uint32_t v, const float (&pr)[2][4], float (&o)[NF][4], int lane)
{
    constexpr int pitch = Geo<T, DP>::kPitchV;
    bool bad = false;
    const int key = lane >> 1;
    for (int c = lane & 1; c < Geo<T, DP>::kChunks; c += 2) {
        uint32_t w[4];
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(v + key * pitch + c * 16) : "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i)
            bad |= sizeof(T) == 4 ? (w[i] & 0x7FFFFFFFu) >= 0x7F7FF000u
                                  : (w[i] & 0x7F800000u) == 0x7F800000u || (w[i] & 0x7F80u) == 0x7F80u;
    }
    uint32_t rows = __ballot_sync(0xffffffffu, bad);
    while (rows) {
        const int kk = (__ffs(rows) - 1) >> 1;
        rows &= ~(3u << (2 * kk));
        const int owner = (lane & ~3) | ((kk & 7) >> 1);
        const float pa0 = __shfl_sync(0xffffffffu, pr[0][0], owner), pa1 = __shfl_sync(0xffffffffu, pr[0][1], owner);
        const float pb0 = __shfl_sync(0xffffffffu, pr[0][2], owner), pb1 = __shfl_sync(0xffffffffu, pr[0][3], owner);
        const float pc0 = __shfl_sync(0xffffffffu, pr[1][0], owner), pc1 = __shfl_sync(0xffffffffu, pr[1][1], owner);
        const float pd0 = __shfl_sync(0xffffffffu, pr[1][2], owner), pd1 = __shfl_sync(0xffffffffu, pr[1][3], owner);
        const float pu = kk < 8 ? (kk & 1 ? pa1 : pa0) : (kk & 1 ? pc1 : pc0);
        const float pl = kk < 8 ? (kk & 1 ? pb1 : pb0) : (kk & 1 ? pd1 : pd0);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int e = f * 8 + 2 * (lane & 3);
            float x0, x1;
            if (sizeof(T) == 2) {
                uint32_t w;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(chunk_at<DP>(v, kk, f) + 4 * (lane & 3)) : "memory");
                x0 = __uint_as_float(w << 16);
                x1 = __uint_as_float(w & 0xFFFF0000u);
            } else {
                asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(x0), "=f"(x1) : "r"(v + kk * pitch + e * 4) : "memory");
            }
            if (pu > 0.f) { o[f][0] = fmaf(pu, x0, o[f][0]); o[f][1] = fmaf(pu, x1, o[f][1]); }
            if (pl > 0.f) { o[f][2] = fmaf(pl, x0, o[f][2]); o[f][3] = fmaf(pl, x1, o[f][3]); }
        }
        __syncwarp();
        for (int c = lane; c < Geo<T, DP>::kChunks; c += 32)
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v + kk * pitch + c * 16), "r"(0u) : "memory");
        __syncwarp();
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, Smem<T, DP>::kCtas) kv_attention_kernel(const __grid_constant__ AttnParams p)
{
    typedef Geo<T, DP> G;
    typedef Smem<T, DP> S;
    constexpr bool kBf16 = sizeof(T) == 2;
    constexpr int kStages = G::kStages;
    constexpr int NF = DP / 8;                             // 8-feature blocks of the accumulator
    constexpr bool kQRegs = kBf16 && DP <= 128;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long sh_find[kWarps + 2];
    __shared__ int sh_last;
    __shared__ Cursor<kRows, kTile> sh_ld[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    const uint32_t ring = s_addr(smem) + warp * kStages * S::kStage;
    const uint32_t sq = s_addr(smem) + S::kRing;
    float *red = reinterpret_cast<float *>(smem + S::kRing + S::kQ);
    float *red_m = reinterpret_cast<float *>(smem + S::kRing + S::kQ + S::kRed), *red_l = red_m + kWarps * kRows;
    const T *kp = reinterpret_cast<const T *>(p.k), *vp = reinterpret_cast<const T *>(p.v);
    const int P = p.b.page.d, chunks = kBf16 ? p.D / 8 : p.D / 4;

    pdl_wait();
    pdl_trigger();
    typedef RowTile<kRows, kTile> Tile;
    Cursor<kRows, kTile> cur;
    long long per;
    const long long len = p.b.n_seqs <= 128 ? find_piece_warp(p, cur, per, blockIdx.x == 0 && warp == 0)
                                            : find_piece<kRows, kTile, kThreads>(p, cur, per, sh_find);
    if (len == 0) return;

    // -- loads run kStages - 1 tiles ahead of the products, through a cursor of their own (in shared memory: it moves
    //    once a unit); the page of the lane's key is fetched another tile ahead
    Cursor<kRows, kTile> &ld = sh_ld[warp];
    if (lane == 0) ld = cur;
    __syncwarp();
    Tile lt = cur.t;
    int l_i = cur.i, l_h = cur.h;
    const int32_t *l_table = p.b.page_table + (size_t)cur.s * p.b.max_pages;
    long long to_load = len;
    int entry = 0, row_in_page = 0;
    bool see = false;
    auto look_up = [&]() {                                 // lanes l and l + 16: key l of the warp's 16
        const int j = key_tile(lt, l_i) * kTile + warp * kWarpKeys + (lane & 15);
        see = j < lt.hi && (j >= lt.lo || j < lt.s1);
        entry = 0;
        row_in_page = 0;
        if (see) {
            const int pg = fast_div(j, p.b.page);
            row_in_page = j - pg * P;
            entry = __ldg(l_table + pg);
        }
    };
    constexpr int per_row = G::kChunks;                    // lanes (16-byte chunks) a row
    constexpr int rows_at_once = per_row >= 32 ? 1 : 32 / per_row;
    constexpr int reps = per_row >= 32 ? per_row / 32 : 1;
    const int l_row = per_row >= 32 ? 0 : lane / per_row, l_ch = per_row >= 32 ? lane : lane % per_row;
    auto load_tile = [&](int stage) {
        if (to_load > 0) {
            if (see && (unsigned)entry >= (unsigned)p.b.n_pages) {
                see = false;
                if (lane < 16) kv_bad_index(p.b);
            }
            const long long off = see ? (long long)entry * p.b.page_stride + ((long long)l_h * P + row_in_page) * p.D : -1;
            const uint32_t dk = ring + stage * S::kStage, dv = dk + kWarpKeys * G::kPitchK;
            if (p.plain_rows && __all_sync(0xffffffffu, see)) {
                // 16 rows of one page, one after the other, as wide as the stage's
                const long long r0 = __shfl_sync(0xffffffffu, off, 0) + (long long)l_row * DP + l_ch * (16 / (int)sizeof(T));
                const T *ks = kp + r0, *vs = vp + r0;
#pragma unroll
                for (int r = 0; r < kWarpKeys; r += rows_at_once) {
                    const int row = r + l_row;
#pragma unroll
                    for (int x = 0; x < reps; ++x) {
                        const int ch = l_ch + 32 * x, dc = G::kSwizzle ? ch ^ (row & 7) : ch;
                        cp16(dk + row * G::kPitchK + dc * 16, ks + r * DP + x * (512 / (int)sizeof(T)), true);
                        cp16(dv + row * G::kPitchV + dc * 16, vs + r * DP + x * (512 / (int)sizeof(T)), true);
                    }
                }
            } else {
#pragma unroll 2
                for (int r = 0; r < kWarpKeys; r += rows_at_once) {
                    const int row = r + l_row;
                    const long long ro = __shfl_sync(0xffffffffu, off, row);
#pragma unroll
                    for (int x = 0; x < reps; ++x) {
                        const int ch = l_ch + 32 * x;
                        const bool on = ro >= 0 && ch < chunks;
                        const long long src = on ? ro + ch * (16 / (int)sizeof(T)) : 0;
                        const int dc = G::kSwizzle ? ch ^ (row & 7) : ch;
                        cp16(dk + row * G::kPitchK + dc * 16, kp + src, on);
                        cp16(dv + row * G::kPitchV + dc * 16, vp + src, on);
                    }
                }
            }
            if (--to_load > 0) {
                if (++l_i == lt.tiles) {
                    __syncwarp();
                    if (lane == 0) {
                        ld.i = lt.tiles - 1;
                        advance(p, ld);
                    }
                    __syncwarp();
                    lt = ld.t;
                    l_i = 0;
                    l_h = ld.h;
                    l_table = p.b.page_table + (size_t)ld.s * p.b.max_pages;
                }
                look_up();
            }
        }
        cp_commit();
    };
    look_up();
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) load_tile(s);

    const long long piece_end = cur.at + len;
    int stage = 0;
    long long at = cur.at;
    while (at < piece_end) {
        // ---- a unit, or the part of it in this piece
        const int begin_tile = cur.i;
        const int count = (int)min((long long)(cur.t.tiles - cur.i), piece_end - at);
        const Tile t = cur.t;
        // queries of the tile -> shared memory, zero beyond the rows and features there are
        for (int i = tid; i < kRows * G::kChunks; i += kThreads) {
            const int r = i / G::kChunks, ch = i - r * G::kChunks;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (r < t.rows && ch < chunks) {
                const int row = t.r0 + r, tok = row / p.g, hg = row - tok * p.g;
                x = __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.q) + (int64_t)(cur.start + tok) * p.q_stride +
                                                          (int64_t)(cur.h * p.g + hg) * p.D) + ch);
            }
            const uint32_t a = sq + r * G::kPitchQ + ((G::kSwizzle ? ch ^ (r & 7) : ch) << 4);
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
        }
        __syncthreads();
        uint32_t qf[kQRegs ? DP / 16 : 1][4];
        if constexpr (kQRegs) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) ldsm4(chunk_at<DP>(sq, lane & 15, 2 * ks + (lane >> 4)), qf[ks]);
        }
        // the two rows of this lane: what they see
        int hi2[2], lo2[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int r = min(gid + 8 * x, t.rows - 1), pos = cur.pre + (t.r0 + r) / p.g;
            hi2[x] = p.mask == MRP_ATTN_CAUSAL ? pos + 1 : t.hi;
            lo2[x] = p.window > 0 ? max(0, pos + 1 - p.window) : 0;
        }
        const int i0 = t.r0 / p.g, i1 = (t.r0 + t.rows - 1) / p.g;
        const int all_hi = p.mask == MRP_ATTN_CAUSAL ? cur.pre + i0 + 1 : t.hi;      // all rows see [all_lo, all_hi)
        const int all_lo = p.window > 0 ? max(0, cur.pre + i1 + 1 - p.window) : 0;
        const bool differ = i0 != i1 && (p.mask == MRP_ATTN_CAUSAL || p.window > 0);

        float o[NF][4];
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[f][x] = 0.f;

        for (int n = 0; n < count; ++n) {
            load_tile((stage + kStages - 1) % kStages);
            cp_wait<kStages - 1>();
            __syncwarp();
            const uint32_t sk = ring + stage * S::kStage, sv = sk + kWarpKeys * G::kPitchK;
            const int j0 = key_tile(t, begin_tile + n) * kTile + warp * kWarpKeys;
            float s[2][4];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) s[x][y] = 0.f;
            if constexpr (kBf16) {
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks) {
                    uint32_t b[4], a[4];
                    ldsm4(chunk_at<DP>(sk, ((lane >> 4) << 3) + (lane & 7), 2 * ks + ((lane >> 3) & 1)), b);
                    if constexpr (kQRegs) {
#pragma unroll
                        for (int x = 0; x < 4; ++x) a[x] = qf[ks][x];
                    } else {
                        ldsm4(chunk_at<DP>(sq, lane & 15, 2 * ks + (lane >> 4)), a);
                    }
                    mma16(s[0], a, b[0], b[1]);
                    mma16(s[1], a, b[2], b[3]);
                }
            } else {
                // the tensor pipe cuts its sums off instead of rounding them: 32 products at a time, added here
#pragma unroll 1
                for (int k4 = 0; k4 < DP / 32; ++k4) {
                    float d[2][4];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) d[x][y] = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {          // features 2 tig, 2 tig + 1 stand for k = tig, tig + 4
                        const int at = ((k4 * 4 + i) * 8 + 2 * tig) * 4;
                        float2 qa, qb;
                        asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(qa.x), "=f"(qa.y) : "r"(sq + gid * G::kPitchQ + at) : "memory");
                        asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(qb.x), "=f"(qb.y) : "r"(sq + (gid + 8) * G::kPitchQ + at) : "memory");
                        uint32_t ah[4], al[4];
                        split_tf32(qa.x, ah[0], al[0]);
                        split_tf32(qb.x, ah[1], al[1]);
                        split_tf32(qa.y, ah[2], al[2]);
                        split_tf32(qb.y, ah[3], al[3]);
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            float2 kb;
                            asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(kb.x), "=f"(kb.y) : "r"(sk + (x * 8 + gid) * G::kPitchK + at) : "memory");
                            uint32_t bh[2], bl[2];
                            split_tf32(kb.x, bh[0], bl[0]);
                            split_tf32(kb.y, bh[1], bl[1]);
                            mma8(d[x], al, bh[0], bh[1]);
                            mma8(d[x], ah, bl[0], bl[1]);
                            mma8(d[x], ah, bh[0], bh[1]);
                        }
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) s[x][y] += d[x][y];
                }
            }
            // what a row does not see scores -inf
            const bool whole = j0 >= all_lo && j0 + kWarpKeys <= all_hi;
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    if (!whole) {
                        const int j = j0 + x * 8 + 2 * tig + (y & 1);
                        s[x][y] = sees(j, hi2[y >> 1], lo2[y >> 1], p.sinks) ? s[x][y] : -INFINITY;
                    }
                    top[y >> 1] = fmaxf(top[y >> 1], s[x][y] * p.scale_log2);
                }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 1));
                top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 2));
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float nm = fmaxf(m[x], top[x]);
                    const float c = m[x] == nm ? 1.f : exp2_fast(m[x] - nm);       // (-inf before the first visible key: 0)
                    l[x] *= c;
#pragma unroll
                    for (int f = 0; f < NF; ++f) { o[f][2 * x] *= c; o[f][2 * x + 1] *= c; }
                    m[x] = nm;
                }
            }
            const float mm[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    s[x][y] = exp2_fast(fmaf(s[x][y], p.scale_log2, -mm[y >> 1]));
                    l[y >> 1] += s[x][y];
                }
            if (!whole && differ) patch_nonfinite<T, DP, NF>(sv, s, o, lane);
            if constexpr (kBf16) {
                // probabilities as bf16 hi + lo (2^-17 together): with few rows the second product costs nothing that shows
                uint32_t a[4], al[4];
                split_bf16(s[0][0], s[0][1], a[0], al[0]);
                split_bf16(s[0][2], s[0][3], a[1], al[1]);
                split_bf16(s[1][0], s[1][1], a[2], al[2]);
                split_bf16(s[1][2], s[1][3], a[3], al[3]);
#pragma unroll
                for (int f = 0; f < NF; f += 2) {
                    uint32_t b[4];
                    ldsm4t(chunk_at<DP>(sv, (((lane >> 3) & 1) << 3) + (lane & 7), f + (lane >> 4)), b);
                    mma16(o[f], al, b[0], b[1]);
                    mma16(o[f + 1], al, b[2], b[3]);
                    mma16(o[f], a, b[0], b[1]);
                    mma16(o[f + 1], a, b[2], b[3]);
                }
            } else {
                uint32_t ah[2][4], al[2][4];               // keys 2 tig, 2 tig + 1 stand for k = tig, tig + 4
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    split_tf32(s[x][0], ah[x][0], al[x][0]);
                    split_tf32(s[x][2], ah[x][1], al[x][1]);
                    split_tf32(s[x][1], ah[x][2], al[x][2]);
                    split_tf32(s[x][3], ah[x][3], al[x][3]);
                }
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        float v0, v1;
                        const uint32_t a0 = sv + (x * 8 + 2 * tig) * G::kPitchV + (f * 8 + gid) * 4;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v0) : "r"(a0) : "memory");
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v1) : "r"(a0 + G::kPitchV) : "memory");
                        uint32_t bh[2], bl[2];
                        split_tf32(v0, bh[0], bl[0]);
                        split_tf32(v1, bh[1], bl[1]);
                        mma8(d, al[x], bh[0], bh[1]);
                        mma8(d, ah[x], bl[0], bl[1]);
                        mma8(d, ah[x], bh[0], bh[1]);
                    }
#pragma unroll
                    for (int y = 0; y < 4; ++y) o[f][y] += d[y];
                }
            }
            __syncwarp();
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }

        // ---- the four warps' parts meet
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
            l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
            if (tig == 0) {
                red_m[warp * kRows + gid + 8 * x] = m[x];
                red_l[warp * kRows + gid + 8 * x] = l[x];
            }
#pragma unroll
            for (int f = 0; f < NF; ++f)
                *reinterpret_cast<float2 *>(red + (size_t)(warp * kRows + gid + 8 * x) * S::kRedPitch + f * 8 + 2 * tig) =
                    make_float2(o[f][2 * x], o[f][2 * x + 1]);
        }
        __syncthreads();
        const bool whole_unit = count == t.tiles;
        const int slot = 2 * blockIdx.x + (begin_tile == 0 ? 1 : 0);
        constexpr int F4 = DP / 4;
        auto put = [&](int r, int f4, float4 a, float M, float L) {       // final values of a row's four features
            const int row = t.r0 + r, tok = row / p.g, head = cur.h * p.g + row - tok * p.g;
            const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);   // (NaN goes through)
            a.x *= inv; a.y *= inv; a.z *= inv; a.w *= inv;
            T *dst = reinterpret_cast<T *>(p.out) + (int64_t)(cur.start + tok) * p.out_stride + (int64_t)head * p.D + f4 * 4;
            if (f4 * 4 < p.D) {
                if constexpr (kBf16) {
                    const __nv_bfloat162 x0 = __floats2bfloat162_rn(a.x, a.y), x1 = __floats2bfloat162_rn(a.z, a.w);
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&x0), *reinterpret_cast<const uint32_t *>(&x1));
                } else {
                    *reinterpret_cast<float4 *>(dst) = a;
                }
            }
            if (f4 == 0 && p.lse)
                p.lse[(int64_t)(cur.start + tok) * p.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
        };
        for (int i = tid; i < t.rows * F4; i += kThreads) {
            const int r = i / F4, f4 = i - r * F4;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red_m[w * kRows + r]);
            float L = 0.f;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float mw = red_m[w * kRows + r];
                const float c = mw == -INFINITY ? 0.f : exp2_fast(mw - M);
                if (mw == -INFINITY && red_l[w * kRows + r] == 0.f) continue;        // saw nothing
                const float4 x = *reinterpret_cast<const float4 *>(red + (size_t)(w * kRows + r) * S::kRedPitch + f4 * 4);
                L = fmaf(c, red_l[w * kRows + r], L);
                a.x = fmaf(c, x.x, a.x); a.y = fmaf(c, x.y, a.y); a.z = fmaf(c, x.z, a.z); a.w = fmaf(c, x.w, a.w);
            }
            if (whole_unit) {
                put(r, f4, a, M, L);
            } else {
                __stcg(reinterpret_cast<float4 *>(p.part.o + ((size_t)slot * kRows + r) * DP) + f4, a);
                if (f4 == 0) __stcg(p.part.ml + (size_t)slot * kRows + r, make_float2(M, L));
            }
        }
        if (!whole_unit) {
            // ---- the pieces of a unit meet: the CTA that arrives last joins them in the order of the pieces
            int c0, c1;
            unit_pieces(p, cur, per, c0, c1);
            __syncthreads();
            if (tid == 0) sh_last = arrive_acq_rel(p.part.counters + c0) == c1 - c0;
            __syncthreads();
            if (sh_last) {
                for (int i = tid; i < t.rows * F4; i += kThreads) {
                    const int r = i / F4, f4 = i - r * F4;
                    float M = -INFINITY;
                    for (int c = c0; c <= c1; ++c) M = fmaxf(M, __ldcg(p.part.ml + (size_t)(2 * c + (c == c0)) * kRows + r).x);
                    float L = 0.f;
                    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
                    for (int c = c0; c <= c1; ++c) {
                        const size_t sl = (size_t)(2 * c + (c == c0)) * kRows + r;
                        const float2 ml = __ldcg(p.part.ml + sl);
                        const float4 x = __ldcg(reinterpret_cast<const float4 *>(p.part.o + sl * DP) + f4);
                        if (ml.x == -INFINITY && ml.y == 0.f) continue;
                        const float w = ml.x == -INFINITY ? 0.f : exp2_fast(ml.x - M);
                        L = fmaf(w, ml.y, L);
                        a.x = fmaf(w, x.x, a.x); a.y = fmaf(w, x.y, a.y); a.z = fmaf(w, x.z, a.z); a.w = fmaf(w, x.w, a.w);
                    }
                    put(r, f4, a, M, L);
                }
                if (tid == 0) p.part.counters[c0] = 0;
            }
        }
        // ---- next unit
        at += count;
        if (at < piece_end) {
            cur.i = t.tiles - 1;
            cur.at = at - 1;
            advance(p, cur);
            __syncthreads();               // the queries and the parts of this unit are read
        }
    }
    cp_wait<0>();
}

size_t slot_bytes() { return (size_t)kRows * (256 * 4 + 8); }

template <typename T, int DP>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(kv_attention_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<T, DP>::kTotal);
}
template <typename T, int DP>
cudaError_t launch(Ctx *c, const AttnParams &p, cudaStream_t st)
{
    const int sms = c->sm_count < kKvMaxSm ? c->sm_count : kKvMaxSm;
    cudaError_t e = launch_k(kv_attention_kernel<T, DP>, dim3(sms * Smem<T, DP>::kCtas), dim3(kThreads), Smem<T, DP>::kTotal, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "kv_attention_kernel");
}

}  // namespace

size_t kv_workspace_bytes(const mrp_config &cfg, const mrp_kv_config &kv)
{
    const size_t few = kKvCounterBytes + (size_t)4 * kKvMaxSm * slot_bytes();
    return kv_tc_takes(cfg, kv) && kv_tc_workspace_bytes() > few ? kv_tc_workspace_bytes() : few;
}

cudaError_t kv_attach(Ctx *c)
{
    // (done before the call returns: the caller's stream need not wait for the legacy one)
    cudaError_t e = cudaMemset(c->kv_ws, 0, kKvCounterBytes);
    if (e != cudaSuccess || (e = cudaStreamSynchronize(cudaStreamLegacy)) != cudaSuccess || (e = kv_tc_attach(c)) != cudaSuccess) return e;
    if (c->cfg.dtype == MRP_BF16) {
        if ((e = prepare<__nv_bfloat16, 64>()) != cudaSuccess || (e = prepare<__nv_bfloat16, 128>()) != cudaSuccess) return e;
        return prepare<__nv_bfloat16, 256>();
    }
    if ((e = prepare<float, 64>()) != cudaSuccess || (e = prepare<float, 128>()) != cudaSuccess) return e;
    return prepare<float, 256>();
}

cudaError_t launch_paged_attention(Ctx *c, const mrp_kv_batch &batch, const mrp_module_kv &pages,
                                   const mrp_attention_args &a, cudaStream_t st)
{
    const mrp_kv_config &kv = c->kv;
    AttnParams p;
    p.b.seq_start = batch.seq_start;
    p.b.prefix_len = batch.prefix_len;
    p.b.page_table = batch.page_table;
    p.b.positions = nullptr;
    p.b.n_seqs = batch.n_seqs;
    p.b.n_tokens = batch.n_tokens;
    p.b.n_pages = kv.n_pages;
    p.b.max_pages = kv.max_pages;
    p.b.cap = kv.max_pages * kv.page_size;
    p.b.page = make_fastdiv(kv.page_size);
    p.b.page_stride = kv.page_stride;
    p.b.status = (int32_t *)(c->ws + c->lay.status);
    p.b.user_status = batch.status;
    p.q = a.q; p.k = pages.k; p.v = pages.v; p.out = a.out; p.lse = a.lse;
    p.q_stride = a.q_stride; p.out_stride = a.out_stride;
    p.H = kv.n_heads; p.Hk = kv.n_kv_heads; p.g = kv.n_heads / kv.n_kv_heads; p.D = kv.head_dim;
    p.gdiv = make_fastdiv(p.g);
    p.mask = a.mask; p.window = a.window; p.sinks = a.window > 0 ? a.sinks : 0;
    p.rows_above = 0;
    p.rows_upto = 0x7fffffff;
    p.lead = 0;
    p.scale_log2 = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)kv.head_dim)) * 1.4426950408889634f;
    {
        // a warp's 16 keys lie one after the other in one page, in rows as wide as the kernel's stages
        const int DP = kv.head_dim <= 64 ? 64 : kv.head_dim <= 128 ? 128 : 256;
        p.plain_rows = kv.page_size % kWarpKeys == 0 && kv.head_dim == DP;
    }
    if (c->kv_encode) return launch_paged_attention_tc(c, p, batch, st);
    const size_t slots = (size_t)4 * kKvMaxSm;
    p.part.counters = (int32_t *)c->kv_ws;
    p.part.ml = (float2 *)(c->kv_ws + kKvCounterBytes);
    p.part.o = (float *)(c->kv_ws + kKvCounterBytes + slots * kRows * 8);
    if (c->cfg.dtype == MRP_BF16)
        return kv.head_dim <= 64 ? launch<__nv_bfloat16, 64>(c, p, st)
             : kv.head_dim <= 128 ? launch<__nv_bfloat16, 128>(c, p, st) : launch<__nv_bfloat16, 256>(c, p, st);
    return kv.head_dim <= 64 ? launch<float, 64>(c, p, st)
         : kv.head_dim <= 128 ? launch<float, 128>(c, p, st) : launch<float, 256>(c, p, st);
}

}  // namespace mrp

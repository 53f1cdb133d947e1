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
// f32 on 8 bits: keys and values are exact in bf16, so m16n8k16 with queries and probabilities in three bf16 parts (2^-24): half the
// products, no splits of keys and half the stage.  24 sequences as below, 128 features 143 us (tf32, one part of K and V: 174),
// 256 features 364 (466); 7 of up to 9 tokens behind a window, heads of 72: 35 (38).  What is left is a tile's chain at two CTAs an SM.
//
// What bounds it: the instructions around the products (f32: splitting K and V, three conversions and a subtraction a value and
// row of the tile), not memory.  24 sequences of 200 to 6000 positions, one token each, 32 / 8 heads: bf16 of 128 features in
// pages of 20 rows 100 us (48 for the bytes); f32 107 (48) at 64 features, 184 (97) at 128, 530 (193) at 256.  Two CTAs an SM
// count more than a second stage: f32 of 128 features 235 us with two stages of one CTA.  Rows beyond 16 take a unit per 16.
#include <cuda_fp16.h>

#include <type_traits>

#include "kv_attention.cuh"
#include "kv_q8.cuh"

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
template <int BYTES> __device__ __forceinline__ void cp_some(uint32_t dst, const void *src, int n)     // 4 or 8, of which n are read
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n) : "memory");
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
// The same for 32 bits in three parts: two cut off (so that none becomes infinite), the last rounded: below 2^-24 of x is left out
__device__ __forceinline__ void split3_bf16(float a, float b, uint32_t (&part)[3])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        part[i] = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632);
        a -= __uint_as_float(__float_as_uint(a) & 0xFFFF0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xFFFF0000u);
    }
    const __nv_bfloat162 l = __floats2bfloat162_rn(a, b);
    part[2] = *reinterpret_cast<const uint32_t *>(&l);
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
template <typename T, int DP, int SRC> struct Smem {
    typedef Geo<T, DP> G;
    // f32 on 8 bits: keys and values are exact in bf16, queries and probabilities go in three bf16 parts
    static constexpr bool kThree = sizeof(T) == 4 && SRC == kFromQ8;
    typedef typename std::conditional<kThree, __nv_bfloat16, T>::type Held;        // what a stage holds
    typedef Geo<Held, DP> GH;
    static constexpr int kStage = kWarpKeys * (GH::kPitchK + GH::kPitchV);
    static constexpr int kRedPitch = DP + 4;               // floats
    // 8 bits: a ring of raw stages (codes of K and V, the 4-byte words their scales lie in, the bytes in those), and one
    // stage of values, which at the end of a unit takes the warp's parts
    static constexpr int kLoads = SRC != kFromQ8 ? G::kStages : DP <= 128 ? 3 : 2;
    static constexpr int kRaw = 2 * kWarpKeys * DP + 2 * kWarpKeys * 4 + 2 * kWarpKeys;
    static constexpr int kParts = kRows * kRedPitch * 4;
    static constexpr int kValues = kStage > kParts ? kStage : kParts;
    static constexpr int kWarp = SRC == kFromQ8 ? kLoads * kRaw + kValues : kLoads * kStage;
    static constexpr int kRing = kWarps * kWarp;
    static constexpr int kQPart = kRows * GH::kPitchQ, kQ = (kThree ? 3 : 1) * kQPart;
    static constexpr int kRed = SRC == kFromQ8 ? 0 : kWarps * kParts;
    static constexpr int kMl = 2 * kWarps * kRows * 4;
    static constexpr int kTotal = kRing + kQ + kRed + kMl;
    static constexpr int kCtas = kTotal <= 113 * 1024 ? 2 : 1;
    static_assert(kStage % 32 == 0 && kRaw % 32 == 0 && kValues % 32 == 0, "aligned stages");
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

template <typename T, int DP, int SRC>
__global__ void __launch_bounds__(kThreads, Smem<T, DP, SRC>::kCtas) kv_attention_kernel(const __grid_constant__ AttnParams p)
{
    typedef Geo<T, DP> G;
    typedef Smem<T, DP, SRC> S;
    typedef typename S::Held Held;
    typedef Geo<Held, DP> GH;
    constexpr bool kBf16 = sizeof(T) == 2, kThree = S::kThree;
    constexpr int kStages = S::kLoads;
    constexpr int NF = DP / 8;                             // 8-feature blocks of the accumulator
    constexpr bool kQRegs = kBf16 && DP <= 128;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ long long sh_find[kWarps + 2];
    __shared__ int sh_last;
    __shared__ Cursor<kRows, kTile> sh_ld[kWarps];
    __shared__ float sh_prior[kRows];                      // log-sum-exps to join with
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    const uint32_t ring = s_addr(smem) + warp * S::kWarp;
    const uint32_t sq = s_addr(smem) + S::kRing;
    auto red = [&](int w) {                                // warp w's parts
        return reinterpret_cast<float *>(smem + (SRC == kFromQ8 ? w * S::kWarp + kStages * S::kRaw : S::kRing + S::kQ + w * S::kParts));
    };
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
    int l_i = cur.i, l_h = cur.h, l_start = cur.start;
    const int32_t *l_table = p.b.page_table + (size_t)cur.s * p.b.max_pages;
    long long to_load = len;
    int entry = 0, row_in_page = 0;
    bool see = false;
    auto look_up = [&]() {                                 // lanes l and l + 16: key l of the warp's 16
        const int j = key_tile(lt, l_i) * kTile + warp * kWarpKeys + (lane & 15);
        see = j < lt.hi && (j >= lt.lo || j < lt.s1);
        entry = 0;
        row_in_page = 0;
        if (SRC == kFromRows) {
            entry = l_start + j;
        } else if (see) {
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
            if (SRC != kFromRows && see && (unsigned)entry >= (unsigned)p.b.n_pages) {
                see = false;
                if (lane < 16) kv_bad_index(p.b);
            }
            if constexpr (SRC == kFromRows) {
                const uint32_t dk = ring + stage * S::kStage, dv = dk + kWarpKeys * G::kPitchK;
                const long long ko = see ? (long long)entry * p.k_stride + l_h * p.D : -1, vo = see ? (long long)entry * p.v_stride + l_h * p.D : -1;
#pragma unroll 2
                for (int r = 0; r < kWarpKeys; r += rows_at_once) {
                    const int row = r + l_row;
                    const long long rk = __shfl_sync(0xffffffffu, ko, row), rv = __shfl_sync(0xffffffffu, vo, row);
#pragma unroll
                    for (int x = 0; x < reps; ++x) {
                        const int ch = l_ch + 32 * x, dc = G::kSwizzle ? ch ^ (row & 7) : ch;
                        const bool on = rk >= 0 && ch < chunks;
                        cp16(dk + row * G::kPitchK + dc * 16, kp + (on ? rk + ch * (16 / (int)sizeof(T)) : 0), on);
                        cp16(dv + row * G::kPitchV + dc * 16, vp + (on ? rv + ch * (16 / (int)sizeof(T)) : 0), on);
                    }
                }
            } else if constexpr (SRC == kFromQ8) {
                const uint32_t raw = ring + stage * S::kRaw, words = raw + 2 * kWarpKeys * DP;
                const uint8_t *kc = reinterpret_cast<const uint8_t *>(p.k), *vc = reinterpret_cast<const uint8_t *>(p.v);
                const long long off = see ? (long long)entry * p.b.page_stride + ((long long)l_h * P + row_in_page) * p.D : -1;
                constexpr int lanes = DP / 8;              // lanes (8 codes) a row
                const int c_row = lane / lanes, c_ch = lane % lanes;
#pragma unroll 2
                for (int r = 0; r < kWarpKeys; r += 32 / lanes) {
                    const int row = r + c_row;
                    const long long ro = __shfl_sync(0xffffffffu, off, row);
                    const bool on = ro >= 0 && c_ch * 8 < p.D;
                    cp_some<8>(raw + row * DP + c_ch * 8, kc + (on ? ro + c_ch * 8 : 0), on ? 8 : 0);
                    cp_some<8>(raw + (kWarpKeys + row) * DP + c_ch * 8, vc + (on ? ro + c_ch * 8 : 0), on ? 8 : 0);
                }
                // lane l: the key's scale of K (l < 16) or V, in the aligned word it lies in (no byte beyond the scales is read)
                const long long so = see ? ((long long)entry * p.Hk + l_h) * P + row_in_page : 0, word = so & ~3ll;
                cp_some<4>(words + lane * 4, (lane < 16 ? p.k_scale : p.v_scale) + word, see ? (int)min(4ll, (long long)p.scale_bytes - word) : 0);
                asm volatile("st.shared.u8 [%0], %1;" ::"r"(words + 2 * kWarpKeys * 4 + lane), "r"((uint32_t)(so & 3)) : "memory");
            } else {
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
                    l_start = ld.start;
                    l_table = p.b.page_table + (size_t)ld.s * p.b.max_pages;
                }
                look_up();
            }
        }
        cp_commit();
    };
    // 8 bits: a landed raw stage -> values, as a stage of the other kinds holds them
    auto to_values = [&](uint32_t raw, uint32_t sk) {
        const uint32_t sv = sk + kWarpKeys * GH::kPitchK, words = raw + 2 * kWarpKeys * DP;
        constexpr int lanes = DP / 8;
        uint32_t at, sc;                                   // of row `lane`: 0 .. 15 keys, then values
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(at) : "r"(words + 2 * kWarpKeys * 4 + lane) : "memory");
        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(sc) : "r"(words + lane * 4 + at) : "memory");
        const float own = q8_factor(sc);
#pragma unroll 2
        for (int i = lane; i < 2 * kWarpKeys * lanes; i += 32) {
            const int row = i / lanes, ch = i % lanes, key = row & 15;
            uint32_t c0, c1;
            asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(c0), "=r"(c1) : "r"(raw + row * DP + ch * 8) : "memory");
            const float f = __shfl_sync(0xffffffffu, own, row);
            const float2 a = q8_values(c0 & 0xFFFFu, f), b = q8_values(c0 >> 16, f), c = q8_values(c1 & 0xFFFFu, f), d = q8_values(c1 >> 16, f);
            const uint32_t to = row < kWarpKeys ? sk + key * GH::kPitchK : sv + key * GH::kPitchV;
            // (exact: four significant bits; below 2^-133 rounded)
            const __nv_bfloat162 w0 = __floats2bfloat162_rn(a.x, a.y), w1 = __floats2bfloat162_rn(b.x, b.y),
                                 w2 = __floats2bfloat162_rn(c.x, c.y), w3 = __floats2bfloat162_rn(d.x, d.y);
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to + ((ch ^ (key & 7)) << 4)), "r"(*reinterpret_cast<const uint32_t *>(&w0)),
                         "r"(*reinterpret_cast<const uint32_t *>(&w1)), "r"(*reinterpret_cast<const uint32_t *>(&w2)),
                         "r"(*reinterpret_cast<const uint32_t *>(&w3)) : "memory");
        }
        __syncwarp();
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
            if constexpr (kThree) {
                uint32_t u[3], w[3];
                split3_bf16(__uint_as_float(x.x), __uint_as_float(x.y), u);
                split3_bf16(__uint_as_float(x.z), __uint_as_float(x.w), w);
#pragma unroll
                for (int y = 0; y < 3; ++y)
                    asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(chunk_at<DP>(sq + y * S::kQPart, r, ch >> 1) + (ch & 1) * 8), "r"(u[y]), "r"(w[y]) : "memory");
            } else {
                const uint32_t a = sq + r * G::kPitchQ + ((G::kSwizzle ? ch ^ (r & 7) : ch) << 4);
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
            }
        }
        if (SRC == kFromRows && p.join && tid < t.rows) {
            const int row = t.r0 + tid, tok = row / p.g;
            sh_prior[tid] = p.lse[(int64_t)(cur.start + tok) * p.H + cur.h * p.g + row - tok * p.g];
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
            const uint32_t sk = SRC == kFromQ8 ? ring + kStages * S::kRaw : ring + stage * S::kStage, sv = sk + kWarpKeys * GH::kPitchK;
            if constexpr (SRC == kFromQ8) to_values(ring + stage * S::kRaw, sk);
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
            } else if constexpr (kThree) {
                // (32 features at a time, added here: see below; the smallest parts first)
#pragma unroll 1
                for (int k2 = 0; k2 < DP / 32; ++k2) {
                    float d[2][4];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) d[x][y] = 0.f;
                    uint32_t b[2][4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) ldsm4(chunk_at<DP>(sk, ((lane >> 4) << 3) + (lane & 7), 4 * k2 + 2 * i + ((lane >> 3) & 1)), b[i]);
#pragma unroll
                    for (int y = 2; y >= 0; --y)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t a[4];
                            ldsm4(chunk_at<DP>(sq + y * S::kQPart, lane & 15, 4 * k2 + 2 * i + (lane >> 4)), a);
                            mma16(d[0], a, b[i][0], b[i][1]);
                            mma16(d[1], a, b[i][2], b[i][3]);
                        }
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int y = 0; y < 4; ++y) s[x][y] += d[x][y];
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
            if (!whole && differ) patch_nonfinite<Held, DP, NF>(sv, s, o, lane);
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
            } else if constexpr (kThree) {
                uint32_t a[3][4];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 4; y += 2) {
                        uint32_t w[3];
                        split3_bf16(s[x][y], s[x][y + 1], w);
#pragma unroll
                        for (int i = 0; i < 3; ++i) a[i][2 * x + (y >> 1)] = w[i];
                    }
#pragma unroll
                for (int f = 0; f < NF; f += 2) {
                    uint32_t b[4];
                    ldsm4t(chunk_at<DP>(sv, (((lane >> 3) & 1) << 3) + (lane & 7), f + (lane >> 4)), b);
                    float d[2][4] = {};
#pragma unroll
                    for (int i = 2; i >= 0; --i) {
                        mma16(d[0], a[i], b[0], b[1]);
                        mma16(d[1], a[i], b[2], b[3]);
                    }
#pragma unroll
                    for (int y = 0; y < 4; ++y) { o[f][y] += d[0][y]; o[f + 1][y] += d[1][y]; }
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
                *reinterpret_cast<float2 *>(red(warp) + (gid + 8 * x) * S::kRedPitch + f * 8 + 2 * tig) =
                    make_float2(o[f][2 * x], o[f][2 * x + 1]);
        }
        __syncthreads();
        const bool whole_unit = count == t.tiles;
        const int slot = 2 * blockIdx.x + (begin_tile == 0 ? 1 : 0);
        constexpr int F4 = DP / 4;
        auto put = [&](int r, int f4, float4 a, float M, float L) {       // final values of a row's four features
            const int row = t.r0 + r, tok = row / p.g, head = cur.h * p.g + row - tok * p.g;
            float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);         // (NaN goes through)
            T *dst = reinterpret_cast<T *>(p.out) + (int64_t)(cur.start + tok) * p.out_stride + (int64_t)head * p.D + f4 * 4;
            JoinWith with = {0.f, 0.f, L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f};
            float4 prior = make_float4(0.f, 0.f, 0.f, 0.f);
            if (SRC == kFromRows && p.join) {
                with = join_with(M, L, sh_prior[r]);
                inv = with.a;
                if (with.b != 0.f && f4 * 4 < p.D) {
                    if constexpr (kBf16) {
                        const uint2 w = *reinterpret_cast<const uint2 *>(dst);
                        prior = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
                    } else {
                        prior = *reinterpret_cast<const float4 *>(dst);
                    }
                    prior.x *= with.b; prior.y *= with.b; prior.z *= with.b; prior.w *= with.b;
                }
            }
            a.x = fmaf(a.x, inv, prior.x); a.y = fmaf(a.y, inv, prior.y); a.z = fmaf(a.z, inv, prior.z); a.w = fmaf(a.w, inv, prior.w);
            if (f4 * 4 < p.D) {
                if constexpr (kBf16) {
                    const __nv_bfloat162 x0 = __floats2bfloat162_rn(a.x, a.y), x1 = __floats2bfloat162_rn(a.z, a.w);
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&x0), *reinterpret_cast<const uint32_t *>(&x1));
                } else {
                    *reinterpret_cast<float4 *>(dst) = a;
                }
            }
            if (f4 == 0 && p.lse)
                p.lse[(int64_t)(cur.start + tok) * p.H + head] = with.lse;
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
                const float4 x = *reinterpret_cast<const float4 *>(red(w) + r * S::kRedPitch + f4 * 4);
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

// Whether packed sequences go without tiles of 128 rows, by the longest as far as the host knows it.  The short kernel takes a chunk of 64
// keys after the other and shares nothing between its CTAs of 64 rows, so a second chunk is what makes it the slower one, and not the
// rows (us in a graph, short / 128-row tiles, n tokens a sequence):
//   one chunk      40 sequences, 32 / 8 heads of 128: n 32 17.6 / 24.9, n 64 30.4 / 41.0; 16 / 8: n 64 19.1 / 27.3; 8 / 1: n 64 12.0 / 18.8
//                  (16 whole blocks, 32 / 8, n 64: 16.9 / 15.7, a wave and a bit of three CTAs an SM; ragged prompts 11.3 / 16.6)
//   half a second  heads of 64: 40, 32 / 8, n 96 32.2 / 42.6, whole blocks 36.1 / 38.6; of 128, where the mask is causal (the first rows skip the
//                  second chunk) and sequences many: 40, 32 / 8 54.3 / 65.1, 16 / 8 32.0 / 39.5, one 11.6 / 10.8; whole blocks 62.3 / 57.5
//   two            40, 32 / 8, n 128 77.7 / 69.3; 16, 16 / 8 23.6 / 20.5
//   heads of 256   one CTA an SM: 16, 16 / 4, n 16 10.9 / 14.8, n 32 (a wave) 12.2 / 16.8, 40 (more) 31.5 / 28.8
// Over the 784 batches measured (1 to 100 sequences, equal or ragged lengths) it costs 1 % over always taking the better one; the dearest
// choices are 100 of n 85, 15 / 5 heads of 80, 53.1 / 47.0, and, not made, 100 ragged of up to 128, 8 / 8, 37.7 / 57.8.
bool packed_short(const Ctx *c, const AttnParams &p, const mrp_kv_batch &batch)
{
    const long long units = (long long)batch.n_seqs * p.Hk, groups = ((long long)batch.max_new * p.g + 63) / 64;
    if (p.D > 128) return batch.max_new <= 64 && (groups <= 1 || units * groups <= c->sm_count);
    return batch.max_new <= 64 || (batch.max_new <= 96 && (p.D <= 64 || (p.mask == MRP_ATTN_CAUSAL && 2 * units > c->sm_count)));
}

size_t slot_bytes() { return (size_t)kRows * (256 * 4 + 8); }

template <typename T, int DP, int SRC>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(kv_attention_kernel<T, DP, SRC>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<T, DP, SRC>::kTotal);
}
template <typename T>
cudaError_t prepare()
{
    cudaError_t all[] = {prepare<T, 64, kFromPages>(), prepare<T, 128, kFromPages>(), prepare<T, 256, kFromPages>(),
                         prepare<T, 64, kFromRows>(), prepare<T, 128, kFromRows>(), prepare<T, 256, kFromRows>(),
                         prepare<T, 64, kFromQ8>(), prepare<T, 128, kFromQ8>(), prepare<T, 256, kFromQ8>()};
    for (cudaError_t one : all)
        if (one != cudaSuccess) return one;
    return cudaSuccess;
}
template <typename T, int DP, int SRC>
cudaError_t launch(Ctx *c, const AttnParams &p, cudaStream_t st)
{
    const int sms = c->sm_count < kKvMaxSm ? c->sm_count : kKvMaxSm;
    cudaError_t e = launch_k(kv_attention_kernel<T, DP, SRC>, dim3(sms * Smem<T, DP, SRC>::kCtas), dim3(kThreads), Smem<T, DP, SRC>::kTotal, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "kv_attention_kernel");
}
template <int SRC>
cudaError_t launch(Ctx *c, AttnParams &p, cudaStream_t st)
{
    const size_t slots = (size_t)4 * kKvMaxSm;
    p.part.counters = (int32_t *)c->kv_ws;
    p.part.ml = (float2 *)(c->kv_ws + kKvCounterBytes);
    p.part.o = (float *)(c->kv_ws + kKvCounterBytes + slots * kRows * 8);
    if (c->cfg.dtype == MRP_BF16)
        return p.D <= 64 ? launch<__nv_bfloat16, 64, SRC>(c, p, st)
             : p.D <= 128 ? launch<__nv_bfloat16, 128, SRC>(c, p, st) : launch<__nv_bfloat16, 256, SRC>(c, p, st);
    return p.D <= 64 ? launch<float, 64, SRC>(c, p, st)
         : p.D <= 128 ? launch<float, 128, SRC>(c, p, st) : launch<float, 256, SRC>(c, p, st);
}

// what does not depend on where keys and values lie
AttnParams attn_params(Ctx *c, const mrp_kv_batch &batch, const mrp_attention_args &a)
{
    const mrp_kv_config &kv = c->kv;
    AttnParams p = {};
    p.b = kv_batch_of(c, batch);
    p.q = a.q; p.out = a.out; p.lse = a.lse;
    p.q_stride = a.q_stride; p.out_stride = a.out_stride;
    p.H = kv.n_heads; p.Hk = kv.n_kv_heads; p.g = kv.n_heads / kv.n_kv_heads; p.D = kv.head_dim;
    p.gdiv = make_fastdiv(p.g);
    p.mask = a.mask; p.window = a.window; p.sinks = a.window > 0 ? a.sinks : 0;
    if (a.mask == MRP_ATTN_PREFIX) p.b.beyond = 0x7fffffff - p.b.cap;      // (the new tokens' own keys lie elsewhere)
    p.rows_upto = 0x7fffffff;
    p.scale_log2 = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)kv.head_dim)) * 1.4426950408889634f;
    return p;
}

}  // namespace

static size_t workspace_for(bool large_tiles)
{
    const size_t few = kKvCounterBytes + (size_t)4 * kKvMaxSm * slot_bytes();
    return large_tiles && kv_tc_workspace_bytes() > few ? kv_tc_workspace_bytes() : few;
}
size_t kv_workspace_bytes(const mrp_config &cfg, const mrp_kv_config &kv) { return workspace_for(kv_tc_any(cfg, kv)); }
// Packed attention alone has large tiles on a geometry whose pages have none: what is smaller serves everything else.
size_t kv_workspace_least(const mrp_config &cfg, const mrp_kv_config &kv) { return workspace_for(kv_tc_takes(cfg, kv)); }
static bool large_tiles_fit(const Ctx *c) { return c->kv_ws_bytes >= kv_tc_workspace_bytes(); }

cudaError_t kv_attach(Ctx *c)
{
    // (done before the call returns: the caller's stream need not wait for the legacy one)
    cudaError_t e = cudaMemset(c->kv_ws, 0, kKvCounterBytes);
    if (e != cudaSuccess || (e = cudaStreamSynchronize(cudaStreamLegacy)) != cudaSuccess || (e = kv_tc_attach(c)) != cudaSuccess) return e;
    return c->cfg.dtype == MRP_BF16 ? prepare<__nv_bfloat16>() : prepare<float>();
}

cudaError_t launch_paged_attention(Ctx *c, const mrp_kv_batch &batch, const mrp_module_kv &pages,
                                   const mrp_attention_args &a, cudaStream_t st)
{
    const mrp_kv_config &kv = c->kv;
    AttnParams p = attn_params(c, batch, a);
    p.k = pages.k; p.v = pages.v;
    {
        // a warp's 16 keys lie one after the other in one page, in rows as wide as the kernel's stages
        const int DP = kv.head_dim <= 64 ? 64 : kv.head_dim <= 128 ? 128 : 256;
        p.plain_rows = kv.page_size % kWarpKeys == 0 && kv.head_dim == DP;
    }
    return kv_tc_takes(c->cfg, kv) ? launch_paged_attention_tc(c, p, batch, st) : launch<kFromPages>(c, p, st);
}

cudaError_t launch_paged_attention_q8(Ctx *c, const mrp_kv_batch &batch, const mrp_kv_pool_q8 &pool,
                                      const mrp_attention_args &a, cudaStream_t st)
{
    AttnParams p = attn_params(c, batch, a);
    p.k = pool.k; p.v = pool.v;
    p.k_scale = pool.k_scale; p.v_scale = pool.v_scale;
    p.scale_bytes = (int64_t)c->kv.n_pages * c->kv.n_kv_heads * c->kv.page_size;
    return kv_tc_takes_q8(c->cfg, c->kv) && large_tiles_fit(c) ? launch_paged_attention_q8_tc(c, p, batch, st) : launch<kFromQ8>(c, p, st);
}

cudaError_t launch_packed_attention(Ctx *c, const mrp_kv_batch &batch, const mrp_packed_kv &kv, const mrp_attention_args &a, cudaStream_t st)
{
    AttnParams p = attn_params(c, batch, a);
    p.b.prefix_len = nullptr;
    p.b.cap = 0x7fffffff;
    p.k = kv.k; p.v = kv.v;
    p.k_stride = kv.k_stride; p.v_stride = kv.v_stride;
    p.join = kv.join != 0;
    if (!kv_tc_takes_rows(c->cfg, c->kv, kv)) return launch<kFromRows>(c, p, st);
    if (packed_short(c, p, batch)) return launch_packed_attention_short(c, p, batch, st);
    return large_tiles_fit(c) ? launch_packed_attention_tc(c, p, batch, st) : launch<kFromRows>(c, p, st);
}

}  // namespace mrp

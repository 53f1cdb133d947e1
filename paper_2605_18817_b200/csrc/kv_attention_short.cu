// Attention of packed rows over each other where sequences are short (the blocks of block diffusion, short prompts), bf16.
//
// The mathematics are those of kv_attention.cu: running maximum (raised only by more than 2^8), scores, probabilities and sums in fp32.
// A sequence of some dozens of tokens is bound by its chain of loads, products and stores, not by any rate, so the work is
// spread as wide as it goes and joined nowhere: a CTA has 64 query rows (row r = token r / g, head r % g) of one sequence and key
// head, a warp 16 of them, which it takes from the scores to the output in registers (mma.sync m16n8k16); keys and values go
// through shared memory in chunks of 64 (cp.async, two stages), and three CTAs share an SM.
// Longer sequences are served rightly too, a chunk after the other; the 128-row tiles (kv_attention_tc.cu) do it faster.  The
// whole call, with joining: 32 blocks of 4, 32 / 8 heads, 8.8 us (128-row tiles 19.0); 12 blocks of 32, 16 / 8 heads, 9.4
// (12.1); 40 prompts of up to 70 tokens, 15 / 5 heads of 80, 17.8 (24.5).
//
// Keys that no row of the CTA sees (behind the sequence's end or the diagonal, before the window) are not read and count as zeros: 0 *
// NaN must not reach a product.  A V row with a value that is not finite that some rows of the CTA see and others do not is zeroed in
// shared memory, and the rows that see it are NaN in all features.
#include "kv_attention.cuh"

namespace mrp {
namespace {

constexpr int kShortThreads = 128;
constexpr int kShortRows = 64, kChunk = 64;                // query rows of a CTA, keys of a chunk
constexpr float kShortLazy = 8.f;                          // log2 of the growth a running maximum may lag behind

struct ShortParams {
    AttnParams a;
    int groups;                // CTAs a sequence and key head (each takes every groups-th 64 rows)
    long long units;           // sequences * key heads * groups
};

template <int DP> struct ShortSmem {
    static constexpr int kPart = kChunk * DP * 2;          // K or V of a chunk
    static constexpr int kTotal = 4 * kPart;
};

__device__ __forceinline__ uint32_t at_smem(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int DP> __device__ __forceinline__ uint32_t row_chunk(uint32_t base, int row, int chunk)     // 16-byte chunks, XOR-swizzled by row
{
    return base + row * (DP * 2) + ((chunk ^ (row & 7)) << 4);
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool on)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void load_matrices(uint32_t a, uint32_t r[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void load_matrices_t(uint32_t a, uint32_t r[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma_bf16(float d[4], const uint32_t a[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_ftz(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b)
{
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&t);
}

// 64 query rows (group rg) of sequence [start, start + n) and key head h
template <int DP>
__device__ __forceinline__ void short_rows(const AttnParams &p, int start, int n, int h, int rg, uint32_t smem, uint32_t *sh_bad)
{
    constexpr int KS = DP / 16, NF = DP / 8, C = DP / 8;   // k-steps, 8-feature blocks, 16-byte chunks of a row
    constexpr bool kQRegs = DP <= 128;
    constexpr int kPart = ShortSmem<DP>::kPart;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    const int rows = n * p.g, r0 = rg * kShortRows, r_end = min(rows, r0 + kShortRows);
    const __nv_bfloat16 *kp = reinterpret_cast<const __nv_bfloat16 *>(p.k) + (int64_t)start * p.k_stride + (int64_t)h * p.D;
    const __nv_bfloat16 *vp = reinterpret_cast<const __nv_bfloat16 *>(p.v) + (int64_t)start * p.v_stride + (int64_t)h * p.D;
    // what the CTA's rows may see: chunks c0 .. c1 - 1, of them those the window or the first tokens reach
    const int i0 = fast_div(r0, p.gdiv), i1 = fast_div(r_end - 1, p.gdiv);
    const int end = p.mask == MRP_ATTN_CAUSAL ? i1 + 1 : n, lo = p.window > 0 ? max(0, i0 + 1 - p.window) : 0;
    const int chunks = (end + kChunk - 1) / kChunk;
    auto next_chunk = [&](int c) {
        for (; c < chunks; ++c)
            if ((c + 1) * kChunk > lo || c * kChunk < p.sinks) break;
        return c;
    };
    auto load = [&](int c, int stage) {
        const uint32_t sk = smem + stage * 2 * kPart, sv = sk + kPart;
        const int fill = min(kChunk, (end - c * kChunk + 15) & ~15) * C;       // (sixteen keys at a time are read)
        for (int i = tid; i < fill; i += kShortThreads) {
            const int row = i / C, ch = i % C, j = c * kChunk + row;
            const bool on = j < end && (j >= lo || j < p.sinks) && ch * 8 < p.D;
            copy16(row_chunk<DP>(sk, row, ch), kp + (on ? (int64_t)j * p.k_stride + ch * 8 : 0), on);
            copy16(row_chunk<DP>(sv, row, ch), vp + (on ? (int64_t)j * p.v_stride + ch * 8 : 0), on);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int c = next_chunk(0);
    if (c < chunks) load(c, 0);

    // ---- the lane's two rows: where they lie, what they see, their queries
    bool live[2];
    int hi_r[2], lo_r[2];
    int64_t q_at[2], o_at[2], l_at[2];
    float prior[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r = r0 + warp * 16 + gid + 8 * x, rr = min(r, rows - 1), tok = fast_div(rr, p.gdiv), head = h * p.g + rr - tok * p.g;
        live[x] = r < rows;
        hi_r[x] = p.mask == MRP_ATTN_CAUSAL ? tok + 1 : n;
        lo_r[x] = p.window > 0 ? max(0, tok + 1 - p.window) : 0;
        q_at[x] = (int64_t)(start + tok) * p.q_stride + (int64_t)head * p.D;
        o_at[x] = (int64_t)(start + tok) * p.out_stride + (int64_t)head * p.D;
        l_at[x] = (int64_t)(start + tok) * p.H + head;
        if (p.join && live[x]) prior[x] = p.lse[l_at[x]];
    }
    const __nv_bfloat16 *q = reinterpret_cast<const __nv_bfloat16 *>(p.q);
    auto query = [&](int ks, uint32_t a[4]) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int x = y & 1, e = ks * 16 + (y >> 1) * 8 + 2 * tig;
            a[y] = live[x] && e < p.D ? __ldg(reinterpret_cast<const uint32_t *>(q + q_at[x] + e)) : 0u;
        }
    };
    uint32_t qf[kQRegs ? KS : 1][4];
    if constexpr (kQRegs) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) query(ks, qf[ks]);
    }
    const bool warp_live = r0 + warp * 16 < rows;
    // what all rows of the warp see
    const int ra = min(r0 + warp * 16, rows - 1), rb = min(r0 + warp * 16 + 15, rows - 1);
    const int all_hi = p.mask == MRP_ATTN_CAUSAL ? fast_div(ra, p.gdiv) + 1 : n, all_lo = p.window > 0 ? max(0, fast_div(rb, p.gdiv) + 1 - p.window) : 0;
    const bool differ = i0 != i1 && (p.mask == MRP_ATTN_CAUSAL || p.window > 0);

    float o[NF][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    bool spoiled[2] = {false, false};      // the row sees a value that is not finite
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int y = 0; y < 4; ++y) o[f][y] = 0.f;

    int stage = 0;
    while (c < chunks) {
        const int after = next_chunk(c + 1);
        if (after < chunks) {
            load(after, stage ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        const uint32_t sk = smem + stage * 2 * kPart, sv = sk + kPart;
        const int j0 = c * kChunk;
        uint32_t bad[2] = {0u, 0u};
        if (differ) {
            // ---- V rows that are not finite: found, zeroed, remembered
            if (tid < 2) sh_bad[tid] = 0u;
            __syncthreads();
            const int key = tid >> 1;      // two threads a key
            bool mine = false;
            for (int ch = tid & 1; ch < C && j0 + key < end; ch += 2) {
                uint32_t w[4];
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(row_chunk<DP>(sv, key, ch)) : "memory");
#pragma unroll
                for (int y = 0; y < 4; ++y) mine |= (w[y] & 0x7F800000u) == 0x7F800000u || (w[y] & 0x7F80u) == 0x7F80u;
            }
            mine = __shfl_xor_sync(0xffffffffu, (int)mine, 1) | mine;
            if (mine && (tid & 1) == 0) atomicOr(&sh_bad[key >> 5], 1u << (key & 31));
            if (mine)
                for (int ch = tid & 1; ch < C; ch += 2)
                    asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(row_chunk<DP>(sv, key, ch)), "r"(0u) : "memory");
            __syncthreads();
            bad[0] = sh_bad[0];
            bad[1] = sh_bad[1];
        } else {
            __syncthreads();
        }
        if (warp_live) {
            const int keys = end - j0;     // of the chunk, or more
            float s[8][4];
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int y = 0; y < 4; ++y) s[t][y] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t a[4];
                if constexpr (kQRegs) {
#pragma unroll
                    for (int y = 0; y < 4; ++y) a[y] = qf[ks][y];
                } else {
                    query(ks, a);
                }
#pragma unroll
                for (int t = 0; t < 8; t += 2) {           // 16 keys
                    if (t * 8 >= keys) break;
                    uint32_t b[4];
                    load_matrices(row_chunk<DP>(sk, t * 8 + ((lane >> 4) << 3) + (lane & 7), 2 * ks + ((lane >> 3) & 1)), b);
                    mma_bf16(s[t], a, b[0], b[1]);
                    mma_bf16(s[t + 1], a, b[2], b[3]);
                }
            }
            const bool whole = j0 >= all_lo && j0 + kChunk <= all_hi;
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    if (!whole) s[t][y] = sees(j0 + t * 8 + 2 * tig + (y & 1), hi_r[y >> 1], lo_r[y >> 1], p.sinks) ? s[t][y] : -INFINITY;
                    top[y >> 1] = fmaxf(top[y >> 1], s[t][y] * p.scale_log2);
                }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 1));
                top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 2));
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] + kShortLazy || top[1] > m[1] + kShortLazy)) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const float nm = fmaxf(m[x], top[x]), e = m[x] == nm ? 1.f : exp2_ftz(m[x] - nm);      // (-inf before the first visible key: 0)
                    l[x] *= e;
#pragma unroll
                    for (int f = 0; f < NF; ++f) { o[f][2 * x] *= e; o[f][2 * x + 1] *= e; }
                    m[x] = nm;
                }
            }
            const float mm[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    s[t][y] = exp2_ftz(fmaf(s[t][y], p.scale_log2, -mm[y >> 1]));
                    l[y >> 1] += s[t][y];
                }
            if (bad[0] | bad[1]) {
#pragma unroll 1
                for (int e = 0; e < kChunk; ++e)
                    if ((bad[e >> 5] >> (e & 31)) & 1u)
#pragma unroll
                        for (int x = 0; x < 2; ++x) spoiled[x] |= sees(j0 + e, hi_r[x], lo_r[x], p.sinks);
            }
            // ---- O += P V, P as bf16 (2^-8 of each at most; the sum takes the unrounded values): half the products of two parts,
            // and what the 128-row tiles do, so that a sequence's precision does not depend on which kernel its batch takes
#pragma unroll
            for (int t = 0; t < 8; t += 2) {
                if (t * 8 >= keys) break;
                const uint32_t a[4] = {two_bf16(s[t][0], s[t][1]), two_bf16(s[t][2], s[t][3]), two_bf16(s[t + 1][0], s[t + 1][1]), two_bf16(s[t + 1][2], s[t + 1][3])};
#pragma unroll
                for (int f = 0; f < NF; f += 2) {
                    uint32_t b[4];
                    load_matrices_t(row_chunk<DP>(sv, t * 8 + (((lane >> 3) & 1) << 3) + (lane & 7), f + (lane >> 4)), b);
                    mma_bf16(o[f], a, b[0], b[1]);
                    mma_bf16(o[f + 1], a, b[2], b[3]);
                }
            }
        }
        __syncthreads();                   // the stage is read
        c = after;
        stage ^= 1;
    }

    // ---- the rows, joined with another pass's where wanted
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
        JoinWith w;
        if (p.join) {
            w = join_with(m[x], l[x], prior[x]);
        } else {
            w.a = l[x] > 0.f ? 1.f / l[x] : (l[x] == 0.f ? 0.f : l[x]);        // (NaN goes through)
            w.b = 0.f;
            w.lse = l[x] == 0.f ? -INFINITY : (m[x] + log2f(l[x])) * 0.6931471805599453f;
        }
        if (spoiled[x]) w.a = __int_as_float(0x7FC00000);
        __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(p.out) + o_at[x];
        uint32_t was[NF];                  // all of the row before any of it is written: their latency once
#pragma unroll
        for (int f = 0; f < NF; ++f) was[f] = w.b != 0.f && live[x] && f * 8 + 2 * tig < p.D ? *reinterpret_cast<const uint32_t *>(dst + f * 8 + 2 * tig) : 0u;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int e = f * 8 + 2 * tig;
            if (live[x] && e < p.D)
                *reinterpret_cast<uint32_t *>(dst + e) = w.b != 0.f ? two_bf16(fmaf(__uint_as_float(was[f] << 16), w.b, o[f][2 * x] * w.a),
                                                                               fmaf(__uint_as_float(was[f] & 0xFFFF0000u), w.b, o[f][2 * x + 1] * w.a))
                                                                    : two_bf16(o[f][2 * x] * w.a, o[f][2 * x + 1] * w.a);
        }
        __syncwarp();                      // (all four lanes of the row have read its log-sum-exp)
        if (live[x] && tig == 0 && p.lse) p.lse[l_at[x]] = w.lse;
    }
}

template <int DP>
__global__ void __launch_bounds__(kShortThreads, DP <= 128 ? 3 : 1) kv_attention_short_kernel(const __grid_constant__ ShortParams sp)
{
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ uint32_t sh_bad[2];
    const AttnParams &p = sp.a;
    pdl_wait();
    pdl_trigger();
#pragma unroll 1
    for (long long u = blockIdx.x; u < sp.units; u += gridDim.x) {
        const long long at = div_line(u, sp.groups);
        const int group = (int)(u - at * sp.groups), s = (int)div_line(at, p.Hk), h = (int)(at - (long long)s * p.Hk);
        int start, n, pre;
        if (!kv_sequence(p.b, s, start, n, pre)) {
            if (h == 0 && group == 0 && threadIdx.x == 0) kv_bad_index(p.b);
            continue;
        }
#pragma unroll 1
        for (int rg = group; (long long)rg * kShortRows < (long long)n * p.g; rg += sp.groups) short_rows<DP>(p, start, n, h, rg, at_smem(smem), sh_bad);
    }
}

template <int DP>
cudaError_t launch_short(Ctx *c, const ShortParams &p, cudaStream_t st)
{
    const long long grid = p.units < (1 << 20) ? p.units : 1 << 20;
    cudaError_t e = launch_k(kv_attention_short_kernel<DP>, dim3((unsigned)grid), dim3(kShortThreads), ShortSmem<DP>::kTotal, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "kv_attention_short_kernel");
}

}  // namespace

cudaError_t kv_short_prepare()
{
    cudaError_t e = cudaFuncSetAttribute(kv_attention_short_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, ShortSmem<64>::kTotal);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kv_attention_short_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, ShortSmem<128>::kTotal);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kv_attention_short_kernel<256>, cudaFuncAttributeMaxDynamicSharedMemorySize, ShortSmem<256>::kTotal);
}

cudaError_t launch_packed_attention_short(Ctx *c, const AttnParams &a, const mrp_kv_batch &batch, cudaStream_t st)
{
    ShortParams p;
    p.a = a;
    const long long rows = (long long)batch.max_new * a.g;
    p.groups = (int)(rows <= kShortRows ? 1 : rows >= 64 * kShortRows ? 64 : (rows + kShortRows - 1) / kShortRows);
    p.units = (long long)batch.n_seqs * a.Hk * p.groups;
    return a.D <= 64 ? launch_short<64>(c, p, st) : a.D <= 128 ? launch_short<128>(c, p, st) : launch_short<256>(c, p, st);
}

}  // namespace mrp

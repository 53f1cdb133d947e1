// Query, key and value rows on their way to the cache: per-head RMSNorm, position rotation, the store into pages.
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma;   (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s),  c + i s = exp(2 pi i f)
// with f the fraction of a turn that position p makes in pair (a, b): p * turn_j mod 2^64, turn_j = 2^64 w_j / (2 pi) on
// the host in 64 bits, so the reduction of the angle is one exact integer product however far the position is.  What is left,
// within half a turn either way, is rounded to fp32 for sincospif (2^-25 half turns at most, an angle of 9e-8: about the
// rounding of the sines themselves).
//
// Every element is read once and written once and takes about seven operations: memory bounds it as long as the
// instructions around them stay few.  A warp takes a token (where tokens are few, one of several shares of a token): it
// finds the token's sequence and page, each lane computes the sines and cosines of its own four pairs once (sincospi),
// and the warp goes through the token's heads in units of one kind (queries, keys, values), GL lanes a head, U heads'
// loads in flight.  A lane holds two runs of four features: the two halves of its four pairs (features 4 l.. and rot_dim / 2
// + 4 l.. of the rotated ones), so a rotation needs no other lane's registers; adjacent pairs lie in one run anyway.
// rot_dim / 2 that is no multiple of four splits runs: there the other half of a pair is read again.
// Measured, 32 query and 8 key heads of 128 in bf16 with norms: 16384 tokens 64 us (336 MB: 5.2 TB/s), 24509 tokens with values
// into pages 105 us (602 MB: 5.7 TB/s, 0.89 of a copy); 4 tokens 3.6 us and 128 tokens 4.2 us a launch inside a graph.
#include "kv_attention.cuh"

namespace mrp {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;

struct RowsParams {
    KvBatch b;                 // b.n_seqs < 0: no batch, positions only
    const void *src[3];        // q, k, v rows (nullptr: none)
    void *dst[3];              // q_out, k_out or the pool of keys, the pool of values
    int64_t src_stride[3], dst_stride[3];
    const void *gamma[2];
    int heads[3];
    int to_pages;              // k and v go to the pools
    int D, rot, half, interleaved;
    int tokens, shares;        // warps a token
    int units[3];              // units of U * NG heads: of queries, and keys, and values
    float eps, inv_d;
    uint64_t turn[128];
};

template <typename T> struct Run4;         // four consecutive features
template <> struct Run4<__nv_bfloat16> {
    uint2 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void get(float *f) const
    {
        f[0] = __uint_as_float(r.x << 16); f[1] = __uint_as_float(r.x & 0xFFFF0000u);
        f[2] = __uint_as_float(r.y << 16); f[3] = __uint_as_float(r.y & 0xFFFF0000u);
    }
    __device__ __forceinline__ void put(const float *f)
    {
        const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        r = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint2 *>(p) = r; }
};
template <> struct Run4<float> {
    float4 r;
    __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void get(float *f) const { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
    __device__ __forceinline__ void put(const float *f) { r = make_float4(f[0], f[1], f[2], f[3]); }
    __device__ __forceinline__ void store(float *p) const { *reinterpret_cast<float4 *>(p) = r; }
};
// two fp32 operations in one instruction
__device__ __forceinline__ void mul2(float &a, float &b, float c, float d)
{
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
__device__ __forceinline__ void fma2(float &a, float &b, float c, float d, float e, float f)     // (a, b) * (c, d) + (e, f)
{
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d), "f"(e), "f"(f));
}
__device__ __forceinline__ float one_f(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float one_f(const float *p) { return *p; }

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

enum { kHalves = 0, kAdjacent = 1, kAgain = 2 };         // how pairs lie in a lane

template <typename T, int GL, int U, int MODE>
__global__ void __launch_bounds__(kRowThreads, 4) qk_rows_kernel(const __grid_constant__ RowsParams p)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int gw = blockIdx.x * kRowWarps + (tid >> 5);
    pdl_wait();
    pdl_trigger();
    // a sequence that does not fit is reported even if no row names it
    if (blockIdx.x == 0)
        for (int s = tid; s < p.b.n_seqs; s += kRowThreads) {
            int start, n, pre;
            if (!kv_sequence(p.b, s, start, n, pre)) kv_bad_index(p.b);
        }
    const int t = gw / p.shares, share = gw - t * p.shares;
    if (t >= p.tokens) return;

    // ---- the token: its sequence, position, row in the pools (element offset of head 0's, -1: not stored)
    int pos = 0;
    int64_t page_off = -1;
    if (p.b.n_seqs >= 0) {
        int s = find_sequence(p.b.seq_start, p.b.n_seqs, t, lane);
        int start, n, pre;
        if (s >= p.b.n_seqs || !kv_sequence(p.b, s, start, n, pre) || t < start || t - start >= n) {
            s = scan_sequences(p.b, t, lane);
            if (s < 0) return;
            kv_sequence(p.b, s, start, n, pre);
        }
        pos = pre + (t - start);
        const int pg = fast_div(pos, p.b.page);
        const int entry = __ldg(p.b.page_table + (size_t)s * p.b.max_pages + pg);
        if ((unsigned)entry < (unsigned)p.b.n_pages)
            page_off = (int64_t)entry * p.b.page_stride + (int64_t)(pos - pg * p.b.page.d) * p.D;
        else if (lane == 0)
            kv_bad_index(p.b);
    }
    if (p.b.positions) pos = __ldg(p.b.positions + t);

    // ---- the lane: two runs of four features, its four pairs
    constexpr int NG = 32 / GL;
    const int gl = lane & (GL - 1), grp = lane / GL;
    const int hl = p.half >> 2;                            // lanes whose runs are the two halves of pairs
    const bool mine = gl * 8 < p.D;
    int e0 = gl * 8, e1 = gl * 8 + 4;
    if (MODE == kHalves) {
        e0 = gl < hl ? gl * 4 : p.rot + (gl - hl) * 8;
        e1 = gl < hl ? p.half + gl * 4 : e0 + 4;
    }
    if (!mine) e0 = e1 = 0;                                // (loads features that are there, stores nothing)
    float cs[4], sn[4];
    if (MODE != kAgain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = gl * 4 + i;
            cs[i] = 1.f;
            sn[i] = 0.f;
            if (j < p.half) {
                const uint64_t f = (uint64_t)(int64_t)pos * p.turn[j];
                sincospif((float)(int32_t)(f >> 32) * 4.656612873077393e-10f, &sn[i], &cs[i]);   // 2^-31: half turns
            }
        }
    }

    // ---- the token's heads
    const int64_t head_out = p.to_pages ? (int64_t)p.b.page.d * p.D : p.D;
#pragma unroll 1
    for (int u = share; u < p.units[2]; u += p.shares) {
        const int kind = u < p.units[0] ? 0 : u < p.units[1] ? 1 : 2;
        const int h0 = (u - (kind == 0 ? 0 : p.units[kind - 1])) * U * NG + grp, n = p.heads[kind] - h0;   // heads h0, h0 + NG, ..
        const T *src = reinterpret_cast<const T *>(p.src[kind]) + (int64_t)t * p.src_stride[kind] + (int64_t)h0 * p.D;
        Run4<T> x[U][2];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const T *row = i * NG < n ? src + i * NG * p.D : src - (n < 1 ? (int64_t)h0 * p.D : 0);     // (beyond the heads: one again)
            x[i][0].load(row + e0);
            x[i][1].load(row + e1);
        }
        T *dst = reinterpret_cast<T *>(p.dst[kind]);
        int64_t step = p.D;
        bool store = mine;
        if (kind > 0 && p.to_pages) {
            step = head_out;
            dst += page_off + (int64_t)h0 * step;
            store = mine && page_off >= 0;
        } else {
            dst += (int64_t)t * p.dst_stride[kind] + (int64_t)h0 * step;
        }
        step *= NG;
        if (kind < 2) {
            const T *gm = reinterpret_cast<const T *>(p.gamma[kind]);
            float g[8];
            if (gm) {
                Run4<T> g0, g1;
                g0.load(gm + e0);
                g1.load(gm + e1);
                g0.get(g);
                g1.get(g + 4);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                float f[8], rs = 1.f;
                x[i][0].get(f);
                x[i][1].get(f + 4);
                if (gm) {
                    float s0 = 0.f, s1 = 0.f;
#pragma unroll
                    for (int y = 0; y < 8; y += 2) {
                        float a = f[y], b = f[y + 1];
                        fma2(a, b, a, b, s0, s1);
                        s0 = a;
                        s1 = b;
                    }
                    float ss = mine ? s0 + s1 : 0.f;
#pragma unroll
                    for (int w = GL / 2; w > 0; w >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, w);
                    rs = rsqrtf(fmaf(ss, p.inv_d, p.eps));
#pragma unroll
                    for (int y = 0; y < 8; y += 2) {
                        mul2(f[y], f[y + 1], rs, rs);
                        mul2(f[y], f[y + 1], g[y], g[y + 1]);
                    }
                }
                if (MODE == kHalves) {
                    if (gl < hl) {                         // (other lanes: features that are not rotated)
#pragma unroll
                        for (int y = 0; y < 4; y += 2) {
                            float a = f[y], b = f[y + 1], c = f[y + 4], d = f[y + 5];
                            mul2(a, b, sn[y], sn[y + 1]);                              // x sin
                            mul2(c, d, -sn[y], -sn[y + 1]);                            // - y sin
                            fma2(f[y], f[y + 1], cs[y], cs[y + 1], c, d);
                            fma2(f[y + 4], f[y + 5], cs[y], cs[y + 1], a, b);
                        }
                    }
                } else if (MODE == kAdjacent) {
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (gl * 8 + 2 * y < p.rot) {
                            const float a = f[2 * y], b = f[2 * y + 1];
                            f[2 * y] = fmaf(a, cs[y], -b * sn[y]);
                            f[2 * y + 1] = fmaf(b, cs[y], a * sn[y]);
                        }
                } else if (mine && i * NG < n) {
                    const T *row = src + i * NG * p.D;
#pragma unroll 1
                    for (int y = 0; y < 8; ++y) {
                        const int e = gl * 8 + y;
                        if (e >= p.rot) continue;
                        const bool first = e < p.half;
                        const int pe = first ? e + p.half : e - p.half;
                        const uint64_t fr = (uint64_t)(int64_t)pos * p.turn[first ? e : pe];
                        float s, c;
                        sincospif((float)(int32_t)(fr >> 32) * 4.656612873077393e-10f, &s, &c);
                        const float o = one_f(row + pe) * (gm ? rs * one_f(gm + pe) : 1.f);
                        const float v = one_f(row + e) * (gm ? rs * one_f(gm + e) : 1.f);
                        const float z = fmaf(v, c, (first ? -o : o) * s);
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (q == y) f[q] = z;
                    }
                }
                x[i][0].put(f);
                x[i][1].put(f + 4);
                if (MODE == kAgain) __syncwarp();          // a head read again above is overwritten by its own lanes alone, now
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (store && i * NG < n) {
                x[i][0].store(dst + i * step + e0);
                x[i][1].store(dst + i * step + e1);
            }
    }
}

template <typename T, int GL, int MODE>
cudaError_t launch_rows(Ctx *c, RowsParams &p, cudaStream_t st)
{
    constexpr int U = sizeof(T) == 2 ? 4 : 2, kAtOnce = U * (32 / GL);
    int n = 0;
    for (int k = 0; k < 3; ++k) p.units[k] = n += (p.heads[k] + kAtOnce - 1) / kAtOnce;
    // A warp a token where there are tokens for every warp the GPU holds; with fewer, a token's units are shared out.
    const long long want = (long long)c->sm_count * 32 / p.tokens;
    p.shares = (int)(want < 1 ? 1 : want > n ? n : want);
    const long long warps = (long long)p.tokens * p.shares;
    cudaError_t e = launch_k(qk_rows_kernel<T, GL, U, MODE>, dim3((unsigned)((warps + kRowWarps - 1) / kRowWarps)), dim3(kRowThreads),
                             0, st, !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "qk_rows_kernel");
}
template <typename T, int GL>
cudaError_t launch_rows(Ctx *c, RowsParams &p, cudaStream_t st)
{
    if (p.interleaved) return launch_rows<T, GL, kAdjacent>(c, p, st);
    return (p.half & 3) == 0 ? launch_rows<T, GL, kHalves>(c, p, st) : launch_rows<T, GL, kAgain>(c, p, st);
}
template <typename T>
cudaError_t launch_rows(Ctx *c, RowsParams &p, cudaStream_t st)
{
    return p.D <= 64 ? launch_rows<T, 8>(c, p, st) : p.D <= 128 ? launch_rows<T, 16>(c, p, st) : launch_rows<T, 32>(c, p, st);
}

}  // namespace

cudaError_t launch_qk_rows(Ctx *c, const mrp_kv_batch *batch, const mrp_module_kv *pages, const int32_t *positions,
                           int n_tokens, const mrp_qkv_rows &rows, cudaStream_t st)
{
    const mrp_kv_config &kv = c->kv;
    RowsParams p;
    p.b = KvBatch{};
    p.b.n_seqs = -1;
    p.b.positions = positions;
    if (batch) {
        p.b.seq_start = batch->seq_start;
        p.b.prefix_len = batch->prefix_len;
        p.b.page_table = batch->page_table;
        p.b.n_seqs = batch->n_seqs;
        p.b.user_status = batch->status;
    }
    p.b.n_tokens = n_tokens;
    p.b.n_pages = kv.n_pages;
    p.b.max_pages = kv.max_pages;
    p.b.cap = kv.max_pages * kv.page_size;
    p.b.page = make_fastdiv(kv.page_size);
    p.b.page_stride = kv.page_stride;
    p.b.status = (int32_t *)(c->ws + c->lay.status);
    p.to_pages = pages != nullptr;
    p.src[0] = rows.q; p.src[1] = rows.k; p.src[2] = pages ? rows.v : nullptr;
    p.dst[0] = rows.q_out; p.dst[1] = pages ? pages->k : rows.k_out; p.dst[2] = pages ? pages->v : nullptr;
    p.src_stride[0] = rows.q_stride; p.src_stride[1] = rows.k_stride; p.src_stride[2] = rows.v_stride;
    p.dst_stride[0] = rows.q_out_stride; p.dst_stride[1] = rows.k_out_stride; p.dst_stride[2] = 0;
    p.gamma[0] = rows.gamma_q; p.gamma[1] = rows.gamma_k;
    p.heads[0] = p.src[0] ? kv.n_heads : 0;
    p.heads[1] = p.src[1] ? kv.n_kv_heads : 0;
    p.heads[2] = p.src[2] ? kv.n_kv_heads : 0;
    p.D = kv.head_dim;
    p.rot = kv.rot_dim;
    p.half = kv.rot_dim / 2;
    p.interleaved = kv.rot_interleaved != 0;
    p.tokens = n_tokens;
    p.eps = kv.norm_eps;
    p.inv_d = 1.f / (float)kv.head_dim;
    for (int j = 0; j < p.half; ++j) p.turn[j] = c->kv_turn[j];
    return c->cfg.dtype == MRP_BF16 ? launch_rows<__nv_bfloat16>(c, p, st) : launch_rows<float>(c, p, st);
}

}  // namespace mrp

// Query, key and value rows on their way to the cache: per-head RMSNorm, position rotation, the store into pages.
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma;   (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s),  c + i s = exp(2 pi i f)
// with f the fraction of a turn that position p makes in pair (a, b): p * turn_j mod 2^64, turn_j = 2^64 w_j / (2 pi) on
// the host in 64 bits, so the reduction of the angle is one exact integer product however far the position is.
//
// Every element is read once and written once and takes about seven operations: memory bounds it, as long as the rest
// stays short.  A warp takes one token (or, where tokens are few, one of several shares of a token's heads): it finds
// the token's sequence and page, each lane computes the sines and cosines of its own four pairs once (sincospi), and
// the warp goes through the token's heads, GL lanes a head, U heads' loads in flight.  A lane holds two runs of four
// features: the two halves of its four pairs (features 4 l.. and rot_dim / 2 + 4 l.. of the rotated ones), so a
// rotation needs no other lane's registers; adjacent pairs lie in one run anyway.  rot_dim / 2 that is no multiple of
// four splits runs: there the other half of a pair is read again.
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
__device__ __forceinline__ float one_f(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float one_f(const float *p) { return *p; }

// Sequence of row t: the number of entries of seq_start[1..n_seqs] that are <= t, found by the warp 32 probes at a time.
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

template <typename T, int GL, int U>
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
        const int s = find_sequence(p.b.seq_start, p.b.n_seqs, t, lane);
        int start, n, pre;
        if (s >= p.b.n_seqs || !kv_sequence(p.b, s, start, n, pre) || t < start) return;
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
    const bool halves = !p.interleaved && (p.half & 3) == 0, again = !p.interleaved && !halves;
    const int hl = p.half >> 2;                            // lanes whose runs are the two halves of pairs
    const bool mine = gl * 8 < p.D;
    int e0 = gl * 8, e1 = gl * 8 + 4;
    if (halves) {
        e0 = gl < hl ? gl * 4 : p.rot + (gl - hl) * 8;
        e1 = gl < hl ? p.half + gl * 4 : e0 + 4;
    }
    float cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = gl * 4 + i;                          // (again: computed where it is used)
        cs[i] = 1.f;
        sn[i] = 0.f;
        if (!again && j < p.half) {
            const uint64_t f = (uint64_t)(int64_t)pos * p.turn[j];
            sincospif((float)(int32_t)(f >> 32) * 4.656612873077393e-10f, &sn[i], &cs[i]);   // 2^-31: half turns
        }
    }
    Run4<T> gq[2], gk[2];
    if (mine && p.gamma[0]) {
        gq[0].load(reinterpret_cast<const T *>(p.gamma[0]) + e0);
        gq[1].load(reinterpret_cast<const T *>(p.gamma[0]) + e1);
    }
    if (mine && p.gamma[1]) {
        gk[0].load(reinterpret_cast<const T *>(p.gamma[1]) + e0);
        gk[1].load(reinterpret_cast<const T *>(p.gamma[1]) + e1);
    }

    // ---- the token's heads: queries, then keys, then values
    const int nq = p.heads[0], nqk = nq + p.heads[1], total = nqk + p.heads[2];
    const T *src0 = reinterpret_cast<const T *>(p.src[0]) + (int64_t)t * p.src_stride[0];
    const T *src1 = reinterpret_cast<const T *>(p.src[1]) + (int64_t)t * p.src_stride[1];
    const T *src2 = reinterpret_cast<const T *>(p.src[2]) + (int64_t)t * p.src_stride[2];
    T *dst0 = reinterpret_cast<T *>(p.dst[0]) + (int64_t)t * p.dst_stride[0];
    const int64_t head_out = p.to_pages ? (int64_t)p.b.page.d * p.D : p.D;
    T *dst1 = reinterpret_cast<T *>(p.dst[1]) + (p.to_pages ? page_off : (int64_t)t * p.dst_stride[1]);
    T *dst2 = reinterpret_cast<T *>(p.dst[2]) + page_off;
    const bool store_kv = !p.to_pages || page_off >= 0;
    for (int r0 = share * NG; r0 < total; r0 += p.shares * NG * U) {
        Run4<T> x[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = min(r0 + u * p.shares * NG + grp, total - 1);
            const T *row = r < nq ? src0 + (int64_t)r * p.D : r < nqk ? src1 + (int64_t)(r - nq) * p.D : src2 + (int64_t)(r - nqk) * p.D;
            if (mine) {
                x[u][0].load(row + e0);
                x[u][1].load(row + e1);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + u * p.shares * NG + grp;
            const bool is_q = r < nq, is_v = r >= nqk;
            float f[8];
            x[u][0].get(f);
            x[u][1].get(f + 4);
            const bool norm = (is_q ? p.gamma[0] : p.gamma[1]) != nullptr && !is_v;
            float rs = 1.f;
            if (p.gamma[0] || p.gamma[1]) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
                if (!mine) ss = 0.f;
#pragma unroll
                for (int w = GL / 2; w > 0; w >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, w);
                if (norm) {
                    rs = rsqrtf(fmaf(ss, p.inv_d, p.eps));
                    Run4<T> g0 = is_q ? gq[0] : gk[0], g1 = is_q ? gq[1] : gk[1];
                    float g[8];
                    g0.get(g);
                    g1.get(g + 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] *= rs * g[i];
                }
            }
            if (p.rot > 0 && !is_v) {
                if (halves) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {          // (beyond the rotated features: cosine 1, sine 0, and
                        if (gl < hl) {                     //  whatever their partner is must not come in)
                            const float a = f[i], b = f[4 + i];
                            f[i] = fmaf(a, cs[i], -b * sn[i]);
                            f[4 + i] = fmaf(b, cs[i], a * sn[i]);
                        }
                    }
                } else if (p.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (gl * 8 + 2 * i < p.rot) {
                            const float a = f[2 * i], b = f[2 * i + 1];
                            f[2 * i] = fmaf(a, cs[i], -b * sn[i]);
                            f[2 * i + 1] = fmaf(b, cs[i], a * sn[i]);
                        }
                } else if (mine && r < total) {
                    const T *row = is_q ? src0 + (int64_t)r * p.D : src1 + (int64_t)(r - nq) * p.D;
                    const T *gm = reinterpret_cast<const T *>(is_q ? p.gamma[0] : p.gamma[1]);
#pragma unroll 1
                    for (int i = 0; i < 8; ++i) {
                        const int e = gl * 8 + i;
                        if (e >= p.rot) continue;
                        const bool first = e < p.half;
                        const int pe = first ? e + p.half : e - p.half;
                        const uint64_t fr = (uint64_t)(int64_t)pos * p.turn[first ? e : pe];
                        float s, c;
                        sincospif((float)(int32_t)(fr >> 32) * 4.656612873077393e-10f, &s, &c);
                        const float o = one_f(row + pe) * (norm ? rs * one_f(gm + pe) : 1.f);
                        const float v = one_f(row + e) * (norm ? rs * one_f(gm + e) : 1.f);
                        const float y = fmaf(v, c, (first ? -o : o) * s);
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k == i) f[k] = y;
                    }
                }
            }
            __syncwarp();                  // a head read again above is overwritten by its own lanes alone, now
            if (mine && r < total && (is_q || store_kv)) {
                T *dst = is_q ? dst0 + (int64_t)r * p.D : is_v ? dst2 + (int64_t)(r - nqk) * head_out : dst1 + (int64_t)(r - nq) * head_out;
                if (!is_v) {
                    x[u][0].put(f);
                    x[u][1].put(f + 4);
                }
                x[u][0].store(dst + e0);
                x[u][1].store(dst + e1);
            }
        }
    }
}

template <typename T, int GL>
cudaError_t launch_rows(Ctx *c, const RowsParams &p, cudaStream_t st)
{
    const long long warps = (long long)p.tokens * p.shares;
    cudaError_t e = launch_k(qk_rows_kernel<T, GL, sizeof(T) == 2 ? 4 : 2>, dim3((unsigned)((warps + kRowWarps - 1) / kRowWarps)),
                             dim3(kRowThreads), 0, st, !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "qk_rows_kernel");
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
    // One warp a token where there are tokens for every warp the GPU holds; with fewer, a token's heads are shared out,
    // down to one round of loads a warp.
    {
        const int rows = p.heads[0] + p.heads[1] + p.heads[2], at_once = 32 / (kv.head_dim <= 64 ? 8 : kv.head_dim <= 128 ? 16 : 32);
        const int most = (rows + at_once * 2 - 1) / (at_once * 2);
        const long long want = (long long)c->sm_count * 24 / n_tokens;
        p.shares = (int)(want < 1 ? 1 : want > most ? most : want);
    }
    p.eps = kv.norm_eps;
    p.inv_d = 1.f / (float)kv.head_dim;
    for (int j = 0; j < p.half; ++j) p.turn[j] = c->kv_turn[j];
    const int lanes = kv.head_dim / 8;
    if (c->cfg.dtype == MRP_BF16)
        return lanes <= 8 ? launch_rows<__nv_bfloat16, 8>(c, p, st)
             : lanes <= 16 ? launch_rows<__nv_bfloat16, 16>(c, p, st) : launch_rows<__nv_bfloat16, 32>(c, p, st);
    return lanes <= 8 ? launch_rows<float, 8>(c, p, st)
         : lanes <= 16 ? launch_rows<float, 16>(c, p, st) : launch_rows<float, 32>(c, p, st);
}

}  // namespace mrp

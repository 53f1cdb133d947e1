// Query, key and value rows on their way to the cache: per-head RMSNorm, position rotation, the store into pages.
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma;   (y_a, y_b) <- (y_a c - y_b s, y_b c + y_a s),  c + i s = exp(2 pi i f)
// with f the fraction of a turn that position p makes in pair (a, b): p * turn_j mod 2^64, turn_j = 2^64 w_j / (2 pi) on
// the host in 64 bits, so the reduction of the angle is one exact integer product however far the position is.
//
// Every element is read once and written once and takes about seven operations: memory bounds it.  A head is handled by
// the GL lanes that hold its features, 8 consecutive ones each (one or two 16-byte accesses); the sum of squares is a
// shuffle reduction over them, and a pair's other half comes from another lane's registers by shuffle where rot_dim / 2
// is a multiple of 8, from the same lane where pairs are adjacent, and is read again otherwise.  Sines and cosines (one
// accurate sincospi per pair) depend on the token alone: a CTA computes them once into shared memory for its few tokens
// and uses them for all heads.
#include "kv_attention.cuh"

namespace mrp {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowMaxTokens = 8;           // tokens of a CTA

struct RowsParams {
    KvBatch b;                 // b.n_seqs < 0: no batch, positions only
    const void *src[3];        // q, k, v rows (nullptr: none)
    void *dst[3];              // q_out, k_out or the pool of keys, the pool of values
    int64_t src_stride[3], dst_stride[3];
    const void *gamma[2];
    int heads[3];
    int to_pages;              // k and v go to the pools
    int D, rot, half, interleaved;
    int tokens, per_cta;
    float eps, inv_d;
    uint64_t turn[128];
};

template <typename T> struct Row8;         // 8 features of a lane
template <> struct Row8<__nv_bfloat16> {
    uint4 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float f[8]) const
    {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void put(const float f[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&t);
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = r; }
};
template <> struct Row8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p)
    {
        a = *reinterpret_cast<const float4 *>(p);
        b = *reinterpret_cast<const float4 *>(p + 4);
    }
    __device__ __forceinline__ void get(float f[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void put(const float f[8])
    {
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
    __device__ __forceinline__ void store(float *p) const
    {
        *reinterpret_cast<float4 *>(p) = a;
        *reinterpret_cast<float4 *>(p + 4) = b;
    }
};
__device__ __forceinline__ float one_f(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float one_f(const float *p) { return *p; }

// What a CTA knows of one of its tokens.
struct TokenAt {
    int go;                    // the token is some sequence's (or there is no batch)
    int pos;                   // position to rotate by
    int64_t page_off;          // element offset of its row of head 0 in a pool, or -1: not stored
};

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
__global__ void __launch_bounds__(kRowThreads) qk_rows_kernel(const __grid_constant__ RowsParams p)
{
    extern __shared__ float sh[];          // cos [per_cta][pitch], sin [per_cta][pitch]
    __shared__ TokenAt at[kRowMaxTokens];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int pitch = (p.half + 3) & ~3;
    float *cs = sh, *sn = sh + (size_t)p.per_cta * pitch;
    const int t0 = blockIdx.x * p.per_cta;
    const int nt = min(p.per_cta, p.tokens - t0);
    pdl_wait();
    pdl_trigger();
    for (int i = warp; i < nt; i += kRowThreads / 32) {
        const int t = t0 + i;
        TokenAt a;
        a.go = 1; a.pos = 0; a.page_off = -1;
        if (p.b.n_seqs >= 0) {
            const int s = find_sequence(p.b.seq_start, p.b.n_seqs, t, lane);
            int start = 0, n = 0, pre = 0;
            const bool in = s < p.b.n_seqs && __ldg(p.b.seq_start + s) <= t;
            const bool ok = in && kv_sequence(p.b, s, start, n, pre);
            a.go = ok;
            if (ok) {
                const int place = pre + (t - start);
                a.pos = place;
                const int pg = fast_div(place, p.b.page);
                const int entry = __ldg(p.b.page_table + (size_t)s * p.b.max_pages + pg);
                if ((unsigned)entry < (unsigned)p.b.n_pages)
                    a.page_off = (int64_t)entry * p.b.page_stride + (int64_t)(place - pg * p.b.page.d) * p.D;
                else if (lane == 0)
                    kv_bad_index(p.b);
            }
        }
        if (p.b.positions && a.go) a.pos = __ldg(p.b.positions + t);
        if (lane == 0) at[i] = a;
    }
    // a sequence that does not fit is reported even if no row names it
    if (blockIdx.x == 0)
        for (int s = tid; s < p.b.n_seqs; s += kRowThreads) {
            int start, n, pre;
            if (!kv_sequence(p.b, s, start, n, pre)) kv_bad_index(p.b);
        }
    __syncthreads();
    for (int i = tid; i < nt * p.half; i += kRowThreads) {
        const int tk = i / p.half, j = i - tk * p.half;
        const uint64_t f = (uint64_t)(int64_t)at[tk].pos * p.turn[j];
        float s, c;
        sincospif((float)(int32_t)(f >> 32) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
        cs[tk * pitch + j] = c;
        sn[tk * pitch + j] = s;
    }
    __syncthreads();

    constexpr int NG = kRowThreads / GL;
    const int gl = tid & (GL - 1), e0 = gl * 8;
    const bool mine = e0 < p.D;
    const int per_token = p.heads[0] + p.heads[1] + p.heads[2];
    const int total = nt * per_token;
    const bool aligned = (p.half & 7) == 0;
    const int hc = p.half >> 3;
    for (int r0 = tid / GL; r0 - tid / GL < total; r0 += NG * U) {
        Row8<T> x[U];
        int kind[U], tok[U], head[U];
        bool live[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + u * NG;
            const int rr = min(r, total - 1);
            tok[u] = rr / per_token;
            int h = rr - tok[u] * per_token;
            kind[u] = 0;
            if (h >= p.heads[0]) { h -= p.heads[0]; kind[u] = 1; }
            if (kind[u] == 1 && h >= p.heads[1]) { h -= p.heads[1]; kind[u] = 2; }
            head[u] = h;
            live[u] = r < total && at[tok[u]].go;
            x[u].load(reinterpret_cast<const T *>(p.src[kind[u]]) + (int64_t)(t0 + tok[u]) * p.src_stride[kind[u]] +
                      (int64_t)h * p.D + (mine ? e0 : 0));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kd = kind[u];
            const T *row = reinterpret_cast<const T *>(p.src[kd]) + (int64_t)(t0 + tok[u]) * p.src_stride[kd] + (int64_t)head[u] * p.D;
            float f[8];
            x[u].get(f);
            const T *gm = kd < 2 ? reinterpret_cast<const T *>(p.gamma[kd]) : nullptr;
            // (the shuffles below are executed by all lanes: heads of one warp may be of different kinds)
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
            if (!mine) ss = 0.f;
#pragma unroll
            for (int w = GL / 2; w > 0; w >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, w);
            const float rs = gm ? 1.f / sqrtf(fmaf(ss, p.inv_d, p.eps)) : 1.f;
            if (gm && mine) {
                Row8<T> g;
                float gf[8];
                g.load(gm + e0);
                g.get(gf);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = f[i] * rs * gf[i];
            }
            if (p.rot > 0) {
                const float *c = cs + tok[u] * pitch, *s = sn + tok[u] * pitch;
                if (p.interleaved) {
                    if (kd < 2) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (e0 + 2 * i < p.rot) {
                                const float cc = c[e0 / 2 + i], sc = s[e0 / 2 + i], a = f[2 * i], b = f[2 * i + 1];
                                f[2 * i] = a * cc - b * sc;
                                f[2 * i + 1] = b * cc + a * sc;
                            }
                    }
                } else if (aligned) {
                    const bool first = gl < hc, turned = gl < 2 * hc;
                    const int from = first ? gl + hc : turned ? gl - hc : gl;
                    float o[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = __shfl_sync(0xffffffffu, f[i], from, GL);
                    if (kd < 2 && turned) {
                        const int j0 = first ? e0 : e0 - p.half;
                        const float sg = first ? -1.f : 1.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] = f[i] * c[j0 + i] + sg * o[i] * s[j0 + i];
                    }
                } else if (kd < 2 && mine) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int e = e0 + i;
                        if (e < p.rot) {
                            const bool first = e < p.half;
                            const int pe = first ? e + p.half : e - p.half, j = first ? e : pe;
                            const float y = one_f(row + pe), o = gm ? y * rs * one_f(gm + pe) : y;
                            f[i] = f[i] * c[j] + (first ? -o : o) * s[j];
                        }
                    }
                }
            }
            __syncwarp();                  // the pairs read again above lie in rows this warp alone may overwrite
            if (live[u] && mine) {
                T *dst = reinterpret_cast<T *>(p.dst[kd]);
                int64_t off;
                if (kd > 0 && p.to_pages) {
                    off = at[tok[u]].page_off;
                    if (off < 0) continue;
                    off += (int64_t)head[u] * p.b.page.d * p.D;
                } else {
                    off = (int64_t)(t0 + tok[u]) * p.dst_stride[kd] + (int64_t)head[u] * p.D;
                }
                if (kd < 2) x[u].put(f);
                x[u].store(dst + off + e0);
            }
        }
    }
}

template <typename T, int GL>
cudaError_t launch_rows(Ctx *c, const RowsParams &p, cudaStream_t st)
{
    const size_t smem = (size_t)2 * p.per_cta * ((p.half + 3) & ~3) * sizeof(float);
    const int grid = (p.tokens + p.per_cta - 1) / p.per_cta;
    cudaError_t e = launch_k(qk_rows_kernel<T, GL, sizeof(T) == 2 ? 4 : 2>, dim3(grid), dim3(kRowThreads), smem, st,
                             !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
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
    // One token per CTA until that fills the GPU's residency; beyond it, several share the start-up and the search.
    p.per_cta = n_tokens <= 8 * c->sm_count ? 1 : n_tokens <= 64 * c->sm_count ? 4 : kRowMaxTokens;
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

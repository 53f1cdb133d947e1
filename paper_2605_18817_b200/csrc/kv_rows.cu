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
// Into 8 bits (the largest of a row over the lanes that hold it, codes by cvt.e4m3x2): 7 prompts of 500 to 3500 tokens with their
// queries 81 us (354 MB: 4.4 TB/s), bound by instructions (issue slots 68 % busy, DRAM 47 %); 24 blocks of 4 5.6 us.
#include <cuda_fp16.h>

#include "kv_attention.cuh"
#include "kv_find.cuh"
#include "kv_q8.cuh"

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
    uint8_t *scale[2];         // of keys and values, where the pools hold 8 bits
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

enum { kHalves = 0, kAdjacent = 1, kAgain = 2 };         // how pairs lie in a lane

template <typename T, int GL, int U, int MODE, bool Q8>
__global__ void __launch_bounds__(kRowThreads, 4) qk_rows_kernel(const __grid_constant__ RowsParams p)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int gw = blockIdx.x * kRowWarps + (tid >> 5);
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0) report_sequences(p.b, tid, kRowThreads);
    const int t = gw / p.shares, share = gw - t * p.shares;
    if (t >= p.tokens) return;

    // ---- the token: its sequence, position, row in the pools (element offset of head 0's, -1: not stored)
    int pos = 0;
    int64_t page_off = -1, scale_off = 0;                  // (8 bits: head 0's scale byte)
    if (p.b.n_seqs >= 0) {
        TokenPlace at;
        if (!find_token(p.b, t, lane, at)) return;
        pos = at.pos;
        if (at.page >= 0) {
            page_off = (int64_t)at.page * p.b.page_stride + (int64_t)at.row * p.D;
            if (Q8) scale_off = (int64_t)at.page * p.heads[1] * p.b.page.d + at.row;
        }
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
        const bool codes = Q8 && kind > 0;
        // 8 bits: the row's scale from its largest magnitude, then the lane's codes and the row's byte
        auto put_codes = [&](float *f, int i) {
            uint32_t top = 0;
#pragma unroll
            for (int y = 0; y < 8; ++y) top = max(top, __float_as_uint(f[y]) & 0x7FFFFFFFu);
            if (!mine) top = 0;
#pragma unroll
            for (int w = GL / 2; w > 0; w >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
            const uint32_t sc = q8_scale(top);
            const bool fine = sc != kQ8NaN;
            const float inv = q8_inverse(fine ? sc : 127u);
#pragma unroll
            for (int y = 0; y < 8; ++y) f[y] *= inv;
            if (sc == kQ8Last)                             // (256 * 2^120 would be infinite: the row stays finite)
#pragma unroll
                for (int y = 0; y < 8; ++y) f[y] = fminf(fmaxf(f[y], -240.f), 240.f);
            if (store && i * NG < n) {
                uint8_t *to = reinterpret_cast<uint8_t *>(p.dst[kind]) + page_off + (int64_t)(h0 + i * NG) * head_out;
                *reinterpret_cast<uint32_t *>(to + e0) = fine ? q8_codes(f[0], f[1], f[2], f[3]) : 0u;
                *reinterpret_cast<uint32_t *>(to + e1) = fine ? q8_codes(f[4], f[5], f[6], f[7]) : 0u;
                if (gl == 0) p.scale[kind - 1][scale_off + (int64_t)(h0 + i * NG) * p.b.page.d] = (uint8_t)sc;
            }
        };
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
                if (codes) {
                    put_codes(f, i);
                } else {
                    x[i][0].put(f);
                    x[i][1].put(f + 4);
                }
                if (MODE == kAgain) __syncwarp();          // a head read again above is overwritten by its own lanes alone, now
            }
        }
        if (codes) {
            if (kind == 2) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    float f[8];
                    x[i][0].get(f);
                    x[i][1].get(f + 4);
                    put_codes(f, i);
                }
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (store && i * NG < n) {
                x[i][0].store(dst + i * step + e0);
                x[i][1].store(dst + i * step + e1);
            }
    }
}

template <typename T, int GL, int MODE, bool Q8>
cudaError_t launch_rows(Ctx *c, RowsParams &p, cudaStream_t st)
{
    constexpr int U = sizeof(T) == 2 ? 4 : 2, kAtOnce = U * (32 / GL);
    int n = 0;
    for (int k = 0; k < 3; ++k) p.units[k] = n += (p.heads[k] + kAtOnce - 1) / kAtOnce;
    // A warp a token where there are tokens for every warp the GPU holds; with fewer, a token's units are shared out.
    const long long want = (long long)c->sm_count * 32 / p.tokens;
    p.shares = (int)(want < 1 ? 1 : want > n ? n : want);
    const long long warps = (long long)p.tokens * p.shares;
    cudaError_t e = launch_k(qk_rows_kernel<T, GL, U, MODE, Q8>, dim3((unsigned)((warps + kRowWarps - 1) / kRowWarps)), dim3(kRowThreads),
                             0, st, !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "qk_rows_kernel");
}
template <typename T, int GL, bool Q8>
cudaError_t launch_rows(Ctx *c, RowsParams &p, cudaStream_t st)
{
    if (p.interleaved) return launch_rows<T, GL, kAdjacent, Q8>(c, p, st);
    return (p.half & 3) == 0 ? launch_rows<T, GL, kHalves, Q8>(c, p, st) : launch_rows<T, GL, kAgain, Q8>(c, p, st);
}
template <typename T, bool Q8>
cudaError_t launch_rows(Ctx *c, RowsParams &p, cudaStream_t st)
{
    return p.D <= 64 ? launch_rows<T, 8, Q8>(c, p, st) : p.D <= 128 ? launch_rows<T, 16, Q8>(c, p, st) : launch_rows<T, 32, Q8>(c, p, st);
}

// what does not depend on where keys and values go
void fill_rows(Ctx *c, RowsParams &p, int n_tokens, const mrp_qkv_rows &rows)
{
    const mrp_kv_config &kv = c->kv;
    p.src[0] = rows.q; p.src[1] = rows.k; p.src[2] = p.to_pages ? rows.v : nullptr;
    p.dst[0] = rows.q_out;
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
}

}  // namespace

cudaError_t launch_qk_rows(Ctx *c, const mrp_kv_batch *batch, const mrp_module_kv *pages, const int32_t *positions,
                           int n_tokens, const mrp_qkv_rows &rows, cudaStream_t st)
{
    RowsParams p;
    if (batch) {
        p.b = kv_batch_of(c, *batch);
    } else {
        p.b = KvBatch{};
        p.b.n_seqs = -1;
        p.b.n_tokens = n_tokens;
        p.b.page = make_fastdiv(c->kv.page_size);
        p.b.status = (int32_t *)(c->ws + c->lay.status);
    }
    p.b.positions = positions;
    p.to_pages = pages != nullptr;
    p.scale[0] = p.scale[1] = nullptr;
    fill_rows(c, p, n_tokens, rows);
    p.dst[1] = pages ? pages->k : rows.k_out;
    p.dst[2] = pages ? pages->v : nullptr;
    return c->cfg.dtype == MRP_BF16 ? launch_rows<__nv_bfloat16, false>(c, p, st) : launch_rows<float, false>(c, p, st);
}

cudaError_t launch_qk_rows_q8(Ctx *c, const mrp_kv_batch &batch, const mrp_kv_pool_q8 &pool, const mrp_qkv_rows &rows, cudaStream_t st)
{
    RowsParams p;
    p.b = kv_batch_of(c, batch);
    p.b.positions = batch.positions;
    p.to_pages = 1;
    fill_rows(c, p, batch.n_tokens, rows);
    p.dst[1] = pool.k; p.dst[2] = pool.v;
    p.scale[0] = pool.k_scale; p.scale[1] = pool.v_scale;
    return c->cfg.dtype == MRP_BF16 ? launch_rows<__nv_bfloat16, true>(c, p, st) : launch_rows<float, true>(c, p, st);
}

}  // namespace mrp

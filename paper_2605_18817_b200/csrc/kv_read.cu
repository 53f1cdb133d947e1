// Rows of the 8-bit cache back in the context dtype: row t of the batch is the key and the value at its position.
//
// Every row is read and written once, D + 1 bytes against 2 D or 4 D: the stores bound it.  A warp takes a token (where tokens are
// few, one of several shares of a token), finds its sequence and page, and goes through its rows (keys of all heads, then
// values) in units of U * NG rows, GL lanes a row, 8 features a lane: an 8-byte load, a 16-byte store (f32: two).
// Measured, 8 heads of 128 in bf16, six caches of 4000 to 20000 positions: 86 us, 6.1 TB/s read and written (0.93 of a copy).
#include <cuda_fp16.h>

#include "kv_attention.cuh"
#include "kv_find.cuh"
#include "kv_q8.cuh"

namespace mrp {
namespace {

constexpr int kReadThreads = 256;
constexpr int kReadWarps = kReadThreads / 32;

struct ReadParams {
    KvBatch b;
    PoolQ8 pool;
    void *dst[2];              // keys, values (nullptr: not wanted)
    int64_t stride[2];
    int heads, D;
    int tokens, shares;        // warps a token
    int units[2];              // units of keys, and values
};

__device__ __forceinline__ void put8(__nv_bfloat16 *p, const float2 (&x)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 y = __floats2bfloat162_rn(x[i].x, x[i].y);
        w[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put8(float *p, const float2 (&x)[4])
{
    *reinterpret_cast<float4 *>(p) = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
}

template <typename T, int GL, int U>
__global__ void __launch_bounds__(kReadThreads) kv_read_kernel(const __grid_constant__ ReadParams p)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int gw = blockIdx.x * kReadWarps + (tid >> 5);
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0) report_sequences(p.b, tid, kReadThreads);
    const int t = gw / p.shares, share = gw - t * p.shares;
    if (t >= p.tokens) return;
    TokenPlace at;
    if (!find_token(p.b, t, lane, at)) return;
    const int64_t row = at.page < 0 ? 0 : (int64_t)at.page * p.heads * p.b.page.d + at.row;            // of head 0, among the scales
    const int64_t code = at.page < 0 ? 0 : (int64_t)at.page * p.b.page_stride + (int64_t)at.row * p.D;
    constexpr int NG = 32 / GL;
    const int gl = lane & (GL - 1), grp = lane / GL;
    if (gl * 8 >= p.D) return;                             // (no exchange between lanes below)
#pragma unroll 1
    for (int u = share; u < p.units[1]; u += p.shares) {
        const int kind = u < p.units[0] ? 0 : 1;
        const int h0 = (u - (kind ? p.units[0] : 0)) * U * NG + grp, n = p.heads - h0;                 // heads h0, h0 + NG, ..
        uint2 c[U];
        uint32_t s[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const bool on = i * NG < n && at.page >= 0;
            const int h = on ? h0 + i * NG : 0;
            c[i] = on ? __ldg(reinterpret_cast<const uint2 *>(p.pool.code[kind] + code + (int64_t)h * p.b.page.d * p.D + gl * 8)) : make_uint2(0, 0);
            s[i] = on ? __ldg(p.pool.scale[kind] + row + (int64_t)h * p.b.page.d) : 127u;
        }
        T *dst = reinterpret_cast<T *>(p.dst[kind]) + (int64_t)t * p.stride[kind] + (int64_t)h0 * p.D + gl * 8;
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (i * NG < n) {
                const float f = q8_factor(s[i]);
                const float2 x[4] = {q8_values(c[i].x & 0xFFFFu, f), q8_values(c[i].x >> 16, f),
                                     q8_values(c[i].y & 0xFFFFu, f), q8_values(c[i].y >> 16, f)};
                put8(dst + (int64_t)i * NG * p.D, x);
            }
    }
}

template <typename T, int GL>
cudaError_t launch_read(Ctx *c, ReadParams &p, cudaStream_t st)
{
    constexpr int U = 4, kAtOnce = U * (32 / GL);
    int n = 0;
    for (int k = 0; k < 2; ++k) p.units[k] = n += p.dst[k] ? (p.heads + kAtOnce - 1) / kAtOnce : 0;
    // A warp a token where there are tokens for every warp the GPU holds; with fewer, a token's units are shared out.
    const long long want = (long long)c->sm_count * 64 / p.tokens;
    p.shares = (int)(want < 1 ? 1 : want > n ? n : want);
    const long long warps = (long long)p.tokens * p.shares;
    cudaError_t e = launch_k(kv_read_kernel<T, GL, U>, dim3((unsigned)((warps + kReadWarps - 1) / kReadWarps)), dim3(kReadThreads),
                             0, st, !(c->cfg.flags & MRP_FLAG_NO_PDL), p);
    c->launches = 1;
    return note_err(c, e, "kv_read_kernel");
}
template <typename T>
cudaError_t launch_read(Ctx *c, ReadParams &p, cudaStream_t st)
{
    return p.D <= 64 ? launch_read<T, 8>(c, p, st) : p.D <= 128 ? launch_read<T, 16>(c, p, st) : launch_read<T, 32>(c, p, st);
}

}  // namespace

cudaError_t launch_kv_read_q8(Ctx *c, const mrp_kv_batch &batch, const mrp_kv_pool_q8 &pool, const mrp_kv_rows &rows, cudaStream_t st)
{
    ReadParams p;
    p.b = kv_batch_of(c, batch);
    p.pool = PoolQ8{{pool.k, pool.v}, {pool.k_scale, pool.v_scale}};
    p.dst[0] = rows.k; p.dst[1] = rows.v;
    p.stride[0] = rows.k_stride; p.stride[1] = rows.v_stride;
    p.heads = c->kv.n_kv_heads;
    p.D = c->kv.head_dim;
    p.tokens = batch.n_tokens;
    return c->cfg.dtype == MRP_BF16 ? launch_read<__nv_bfloat16>(c, p, st) : launch_read<float>(c, p, st);
}

}  // namespace mrp

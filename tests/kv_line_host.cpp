// The cut of the line of tiles (kv_attention.cuh), run on the host: which CTA arrives where, when some of them give up part way.
//
// Reads batches from stdin, a line each: rows tile heads g mask window sinks lead ctas seed n (prefix new) * n
// Every CTA's piece is walked as the kernels walk it: arrivals of the units up to a random one (where a wait gives up), the
// others by settle_arrivals.  Prints "cut <units> left <arrivals missing or too many> dirty <counters that are not zero>".
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <math.h>
#include <random>
#include <vector>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
using std::max;
using std::min;

// what of the device's functions the header names
namespace mrp_host {
struct Dim { unsigned x = 0, y = 0, z = 0; };
}
static mrp_host::Dim threadIdx, blockIdx, gridDim;
template <typename T> static T __ldg(const T *p) { return *p; }
template <typename T> static T __ldcg(const T *p) { return *p; }
static inline unsigned __umulhi(unsigned a, unsigned b) { return (unsigned)(((uint64_t)a * b) >> 32); }
static inline int atomicOr(int *p, int v) { const int old = *p; *p |= v; return old; }
template <typename T> static T __shfl_xor_sync(unsigned, T v, int) { return v; }
template <typename T> static T __shfl_up_sync(unsigned, T v, int) { return v; }
template <typename T> static T __shfl_sync(unsigned, T v, int) { return v; }
static inline unsigned __ballot_sync(unsigned, bool x) { return x; }
static inline int __ffs(int x) { return ffs(x); }
static inline void __syncthreads() {}
static inline void __threadfence() {}
static inline int atomicAdd(int *p, int v) { const int old = *p; *p += v; return old; }
static inline float rsqrtf(float x) { return 1.f / sqrtf(x); }
static inline float __uint_as_float(unsigned x) { float f; memcpy(&f, &x, 4); return f; }

#include "kv_attention.cuh"

using namespace mrp;

template <int ROWS, int TILE> static void run(AttnParams p, int ctas, std::mt19937 &rng)
{
    typedef Cursor<ROWS, TILE> C;
    long long total = 0;
    for (int s = 0; s < p.b.n_seqs; ++s) total += sequence_tiles<ROWS, TILE>(p, s, false);
    const long long per = div_line(total + ctas - 1, ctas);
    std::vector<int> counters(ctas + 1, 0), seen(ctas + 1, 0), due(ctas + 1, 0);
    std::vector<C> at(ctas);
    std::vector<long long> end(ctas, 0);
    C c;
    c.s = 0; c.at = c.unit = 0;
    const bool any = total > 0 && open_sequence(p, c);
    for (int k = 0; k < ctas; ++k) {       // the cursor at the start of each piece, a place at a time
        end[k] = min(total, per * (k + 1));
        at[k] = c;
        if (per * k >= total) { at[k].at = end[k]; continue; }
        while (any && c.at < end[k] && c.at + 1 < total) advance(p, c);
    }
    int cut = 0;
    std::vector<int> order(ctas);
    for (int k = 0; k < ctas; ++k) order[k] = k;
    std::shuffle(order.begin(), order.end(), rng);
    for (int k : order) {
        int stop = (int)(rng() % 4);       // units this CTA gets through before a wait gives up (3: all of them)
        if (stop == 3) stop = 1 << 30;
        C w = at[k];
        auto arrive = [&](const C &, int c0, int c1) {
            due[c0] = c1 - c0 + 1;
            ++seen[c0];
            ++cut;
            if (counters[c0]++ == c1 - c0) counters[c0] = 0;
        };
        for (int u = 0; u < stop && w.at < end[k]; ++u) {          // the kernels' loop
            const UnitPart part = unit_part(p, w, end[k]);
            if (part.count > 0 && part.count != w.t.tiles) {
                int c0, c1;
                unit_pieces(p, w, per, c0, c1);
                arrive(w, c0, c1);
            }
            leave_unit(p, w, part.places, end[k]);
        }
        settle_arrivals(p, w, per, end[k], arrive);
    }
    int left = 0, dirty = 0;
    for (int k = 0; k <= ctas; ++k) {
        left += std::abs(seen[k] - due[k]);
        dirty += counters[k] != 0;
    }
    printf("cut %d left %d dirty %d\n", cut, left, dirty);
}

int main()
{
    int rows, tile, heads, g, mask, window, sinks, lead, ctas, n;
    unsigned seed;
    while (scanf("%d %d %d %d %d %d %d %d %d %u %d", &rows, &tile, &heads, &g, &mask, &window, &sinks, &lead, &ctas, &seed, &n) == 11) {
        std::vector<int32_t> pre(n), start(1, 0);
        for (int i = 0, m; i < n; ++i) {
            if (scanf("%d %d", &pre[i], &m) != 2) return 1;
            start.push_back(start.back() + m);
        }
        AttnParams p;
        memset((void *)&p, 0, sizeof p);
        p.b.seq_start = start.data();
        p.b.prefix_len = pre.data();
        p.b.n_seqs = n;
        p.b.n_tokens = start.back();
        p.b.cap = 1 << 30;
        p.Hk = heads; p.g = g; p.H = heads * g;
        p.gdiv = make_fastdiv(g);
        p.mask = mask; p.window = window; p.sinks = window > 0 ? sinks : 0;
        p.rows_upto = 0x7fffffff;
        p.lead = lead;
        std::mt19937 rng(seed);
        if (rows == 16 && tile == 128) run<16, 128>(p, ctas, rng);
        else if (rows == 16) run<16, 64>(p, ctas, rng);
        else if (rows == 128) run<128, 128>(p, ctas, rng);
        else run<256, 128>(p, ctas, rng);
    }
    return 0;
}

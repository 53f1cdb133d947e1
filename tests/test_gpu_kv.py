"""The paged-cache operators (mrp_qk_norm_rotate, mrp_kv_append, mrp_paged_attention) on the GPU against their 64-bit
statements in oracle/kv.py.

Tolerances, from the arithmetic.  u = 2^-24 (fp32), r = 2^-8 (bf16) or u.
  rotate: the sum of squares of D terms (D u relative, halved by the root), three products and the rotation's two products
    and a sum, sines and cosines off by 2^-22 at most (angle 2^-24 half turns * pi, two ulp): (D/2 + 16) u times the
    largest the pair can be, and one rounding r of the result.
  attend: a score of size z = scale sum |q||k| is off by D u z (bf16: exact products summed in fp32) or (D u + 2^-20) z
    (f32: products of split operands, 2^-21 each side), its scaling to base 2 and the exponential add 4 u (|z| + 1): that is the
    relative error of a probability, twice (numerator and sum), with n u from sums over n keys; bf16 rounds a probability
    by r; f32 adds 2^-20 from the split product.  All of it weighs on reach = sum p |v|; then one rounding r of the result.
  lse: the score error plus the relative error of the sum, 4 u |lse| for logarithm and scaling."""
import math

import numpy as np
import pytest
import torch

from oracle import kv as ref

DEV = "cuda:0"
U = 2.0 ** -24
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(TORCH[dtype]).eps / 2


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


class Cache:
    """A pool, a page table in shuffled order and a batch, with NaN wherever no position lies."""

    def __init__(self, dtype, H, Hk, D, P, lens, seed=0, rot=0, extra_rows=0, page_gap=0, interleaved=False, theta=1e4,
                 inv_freq=None, spare_pages=2, max_seqs=None, positions=None):
        from paper_2605_18817_b200 import binding
        self.b, self.dtype, self.H, self.Hk, self.D, self.P, self.lens = binding, dtype, H, Hk, D, P, lens
        dt = TORCH[dtype]
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.rand = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.float32).to(dt)
        need = [max(1, -(-(p + n) // P)) for p, n in lens]
        self.max_pages = max(need) + 1
        n_pages = sum(need) + spare_pages
        order = torch.randperm(n_pages, generator=g, device=DEV).cpu().tolist()
        table = np.full((len(lens), self.max_pages), -12345, np.int32)         # entries of unused pages are never read
        for b, c in enumerate(need):
            table[b, :c] = [order.pop() for _ in range(c)]
        self.table_np = table
        page = Hk * P * D
        stride = page + page_gap
        self.k_pages, self.v_pages = (torch.full((n_pages * stride,), float("nan"), device=DEV, dtype=dt)
                                      .as_strided((n_pages, Hk, P, D), (stride, P * D, D, 1)) for _ in range(2))
        for b, (p, n) in enumerate(lens):
            for j0 in range(0, p + n, P):
                m = min(P, p + n - j0)
                for pool in (self.k_pages, self.v_pages):
                    pool[table[b, j0 // P], :, :m] = self.rand(Hk, m, D)
        starts = np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int32)
        self.T = int(starts[-1]) + extra_rows
        self.start_np, self.pre_np = starts, np.array([p for p, _ in lens], np.int32)
        self.seq_start, self.prefix_len, self.table = (torch.from_numpy(a).to(DEV) for a in (starts, self.pre_np, table))
        self.status = torch.zeros(1, device=DEV, dtype=torch.int32)
        w_lm = torch.zeros((32, 64), device=DEV, dtype=dt)
        self.ctx = binding.mrp_create(64, 64, 32, [], w_lm, max_rows=1, max_seqs=max_seqs or len(lens), block_len=1)
        self.rot, self.interleaved, self.theta, self.inv_freq = rot, interleaved, theta, inv_freq
        binding.mrp_kv_attach(self.ctx, H, Hk, D, P, n_pages, self.max_pages, stride if page_gap else 0, rot, theta, interleaved, inv_freq)
        self.batch = binding.KvBatch(self.seq_start, self.prefix_len, self.table, self.T, max([n for _, n in lens] + [0]), positions, self.status)

    def attend(self, q, out=None, lse=True, **kw):
        out = torch.full((q.shape[0], self.H, self.D), 7.0, device=DEV, dtype=q.dtype) if out is None else out
        lse = torch.full((q.shape[0], self.H), 7.0, device=DEV) if lse else None
        self.b.mrp_paged_attention(self.ctx, self.batch, self.k_pages, self.v_pages, q, out, lse, **kw)
        return out, lse

    def check(self, q, out, lse, mask=0, window=0, sinks=0, scale=0.0):
        torch.cuda.synchronize()
        o, l, reach, size = ref.attention(f64(q), f64(self.k_pages), f64(self.v_pages), self.start_np, self.pre_np, self.table_np,
                                          self.P, mask, window, sinks, scale, out=np.full(q.shape, 7.0))
        rows = np.zeros(q.shape[0], bool)
        for _, s, n, _ in ref.sequences(self.start_np, self.pre_np, q.shape[0], self.max_pages * self.P):
            rows[s:s + n] = True
        n = max(p + m for p, m in self.lens) + 1
        r, split = half_step(self.dtype), 0.0 if self.dtype == "bf16" else 2.0 ** -20
        z = (self.D * U + split) * size + 4 * U * (size + 1)
        p = 2 * z + 2 * n * U + (r if self.dtype == "bf16" else split)
        tol = reach * p[..., None] + r * np.abs(o) + 1e-30
        got = f64(out)
        assert np.isfinite(got).all()
        assert (np.abs(got - o)[rows] <= tol[rows]).all(), (np.abs(got - o) / tol)[rows].max()
        assert (got[~rows] == 7.0).all()
        if lse is not None:
            gl = f64(lse)
            empty = np.isneginf(l)
            assert np.array_equal(np.isneginf(gl), empty)
            assert (got[rows & empty.all(-1)] == 0).all()
            fine = rows[:, None] & ~empty
            lt = z + n * U + 4 * U * (np.abs(l) + 1)
            assert (np.abs(gl - l)[fine] <= lt[fine]).all(), (np.abs(gl - l)[fine] / lt[fine]).max()
            assert (gl[~rows] == 7.0).all()


ATTEND = [
    # dtype, H, Hk, D, P, [(cached, new)], mask, window, sinks
    ("bf16", 4, 2, 128, 16, [(0, 1)], 0, 0, 0),
    ("bf16", 4, 2, 128, 16, [(63, 1)], 0, 0, 0),
    ("bf16", 4, 4, 64, 16, [(64, 1), (65, 1), (0, 1), (15, 1), (16, 1)], 0, 0, 0),
    ("bf16", 16, 2, 128, 32, [(700, 1), (1300, 1), (1, 1)], 0, 0, 0),
    ("bf16", 24, 2, 128, 64, [(200, 3), (511, 2)], 0, 0, 0),                      # 12 heads a key head: rows over two tiles
    ("bf16", 3, 1, 80, 24, [(100, 5), (0, 17), (333, 0), (50, 1)], 0, 0, 0),
    ("bf16", 5, 1, 8, 7, [(20, 2), (13, 1)], 0, 0, 0),
    ("bf16", 8, 8, 256, 16, [(130, 3)], 0, 0, 0),
    ("bf16", 6, 2, 200, 100, [(201, 9), (99, 1)], 1, 0, 0),
    ("bf16", 8, 2, 128, 32, [(300, 16), (17, 16), (0, 16)], 1, 0, 0),
    ("bf16", 8, 2, 128, 32, [(300, 16), (17, 16), (0, 16)], 2, 0, 0),             # the third sees nothing
    ("bf16", 4, 1, 128, 16, [(1000, 4), (30, 4)], 0, 100, 20),
    ("bf16", 4, 1, 128, 16, [(1000, 4), (30, 4)], 0, 1, 0),
    ("bf16", 4, 1, 64, 64, [(1000, 20), (4, 9)], 2, 5, 0),                        # PREFIX and a short window: late tokens see nothing
    ("bf16", 4, 1, 64, 64, [(1000, 20), (0, 9)], 2, 5, 70),
    ("bf16", 4, 2, 128, 128, [(500, 130), (3, 70)], 1, 64, 64),
    ("bf16", 4, 2, 128, 64, [(129, 300), (0, 257)], 0, 0, 0),                     # prompts
    ("bf16", 7, 7, 96, 16, [(37, 150)], 0, 33, 3),
    ("bf16", 16, 4, 128, 1, [(70, 2)], 0, 0, 0),
    ("bf16", 2, 1, 128, 16, [(5, 1)] * 150, 0, 0, 0),                             # more sequences than threads in the cut
    ("bf16", 2, 1, 128, 4096, [(4000, 1), (4096, 30)], 0, 0, 0),
    ("f32", 4, 2, 64, 16, [(200, 1), (0, 1), (77, 3)], 0, 0, 0),
    ("f32", 4, 4, 128, 24, [(130, 2), (515, 1)], 0, 0, 0),
    ("f32", 3, 1, 40, 10, [(90, 8), (0, 3)], 1, 0, 0),
    ("f32", 2, 1, 256, 16, [(150, 20)], 0, 50, 10),
    ("f32", 8, 1, 128, 32, [(33, 40), (0, 40)], 2, 0, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", ATTEND, ids=lambda c: "%s-H%d-%d-D%d-P%d-n%d-m%d-w%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5]), c[6], c[7]))
def test_attention_over_pages(case):
    dtype, H, Hk, D, P, lens, mask, window, sinks = case
    c = Cache(dtype, H, Hk, D, P, lens, seed=H + D + P)
    q = c.rand(c.T, H, D) * 1.5
    out, lse = c.attend(q, mask=mask, window=window, sinks=sinks)
    c.check(q, out, lse, mask, window, sinks)
    again, _ = c.attend(q, mask=mask, window=window, sinks=sinks)
    assert torch.equal(out, again)
    assert int(c.status.item()) == 0


ROTATE = [
    # dtype, T, H, Hk, D, rot, interleaved, norm
    ("bf16", 1, 4, 2, 128, 128, False, True), ("bf16", 33, 16, 8, 128, 64, False, True), ("bf16", 5, 3, 1, 80, 20, False, True),
    ("bf16", 7, 2, 2, 256, 256, True, True), ("bf16", 9, 5, 1, 64, 0, False, True), ("bf16", 3, 1, 1, 8, 8, False, False),
    ("f32", 1300, 2, 1, 128, 128, False, True), ("f32", 31, 6, 2, 72, 36, False, False), ("f32", 10, 4, 4, 256, 200, False, True),
    ("f32", 17, 3, 3, 40, 30, True, True), ("f32", 2, 8, 1, 16, 6, False, True),
]


def rotate_tol(x, gamma, dtype, D, eps=1e-6):
    x = np.asarray(x, np.float64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gamma
    return (D / 2 + 16) * U * 2 * np.abs(x).max(-1, keepdims=True)


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("case", ROTATE, ids=str)
def test_norm_and_rotation(case, packed):
    dtype, T, H, Hk, D, rot, interleaved, norm = case
    c = Cache(dtype, H, Hk, D, 16, [(0, 1)], rot=rot, interleaved=interleaved, theta=5e5)
    rows = c.rand(T, H + 2 * Hk, D)
    q, k = (rows[:, :H], rows[:, H:H + Hk]) if packed else (rows[:, :H].contiguous(), rows[:, H:H + Hk].contiguous())
    gq, gk = (1 + 0.2 * c.rand(D), 1 + 0.2 * c.rand(D)) if norm else (None, None)
    rng = np.random.default_rng(3)
    pos = rng.integers(-5, 2 ** 21, T).astype(np.int32)
    pos[0] = 0
    pos[-1] = 2 ** 31 - 1 if T > 2 else 17
    qo, ko = torch.full((T, H, D), 5.0, device=DEV, dtype=TORCH[dtype]), torch.full((T, Hk, D), 5.0, device=DEV, dtype=TORCH[dtype])
    c.b.mrp_qk_norm_rotate(c.ctx, torch.from_numpy(pos).to(DEV) if rot else None, q, k, qo, ko, gq, gk)
    for x, gm, got in ((q, gq, qo), (k, gk, ko)):
        g64 = None if gm is None else f64(gm)
        want = ref.norm_rotate(f64(x), pos, g64, rot, 5e5, None, interleaved)
        tol = rotate_tol(f64(x), g64, dtype, D) + half_step(dtype) * np.abs(want)
        if T > 2:                                        # the 64-bit angle itself is off by 2^-53 of 2^31 turns
            tol[-1] += 2.0 ** 31 * 2.0 ** -52 * 4 * np.abs(f64(x)[-1]).max() * (1 if g64 is None else 4)
        assert (np.abs(f64(got) - want) <= tol).all(), (np.abs(f64(got) - want) / tol).max()
    # in place, queries alone
    q2 = q.contiguous().clone()
    c.b.mrp_qk_norm_rotate(c.ctx, torch.from_numpy(pos).to(DEV) if rot else None, q2, None, q2, None, gq, None)
    assert torch.equal(q2, qo)


APPEND = [
    ("bf16", 4, 2, 128, 16, [(0, 5), (15, 1), (16, 17), (3, 0), (40, 2)], 128, False, 0),
    ("bf16", 3, 1, 80, 7, [(6, 9), (0, 1)], 20, False, 64),
    ("bf16", 2, 2, 256, 32, [(31, 40)], 256, True, 0),
    ("f32", 4, 1, 64, 24, [(23, 2), (0, 30), (500, 1)], 48, False, 128),
    ("f32", 1, 1, 8, 1, [(2, 3)], 0, False, 0),
    ("bf16", 8, 8, 64, 16, [(i, 1) for i in range(70)], 64, False, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append_to_pages(case):
    dtype, H, Hk, D, P, lens, rot, interleaved, gap = case
    c = Cache(dtype, H, Hk, D, P, lens, seed=1, rot=rot, interleaved=interleaved, extra_rows=3, page_gap=gap)
    rows = c.rand(c.T, H + 2 * Hk, D)
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    gq, gk = 1 + 0.2 * c.rand(D), 1 + 0.2 * c.rand(D)
    k0, v0 = f64(c.k_pages), f64(c.v_pages)
    qo = torch.full((c.T, H, D), 5.0, device=DEV, dtype=TORCH[dtype])
    c.b.mrp_kv_append(c.ctx, c.batch, c.k_pages, c.v_pages, k, v, gk, q, qo, gq)
    pos = np.zeros(c.T, np.int64)
    rowmask = np.zeros(c.T, bool)
    for _, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * P):
        pos[s:s + n] = p + np.arange(n)
        rowmask[s:s + n] = True
    kw = ref.norm_rotate(f64(k), pos, f64(gk), rot, 1e4, None, interleaved)
    qw = ref.norm_rotate(f64(q), pos, f64(gq), rot, 1e4, None, interleaved)
    kp, vp = ref.append(k0, v0, kw, f64(v), c.start_np, c.pre_np, c.table_np, P)
    assert np.array_equal(f64(c.v_pages), vp, equal_nan=True)
    got = f64(c.k_pages)
    written = ~((got == k0) | (np.isnan(got) & np.isnan(k0)))
    assert np.array_equal(np.isnan(got), np.isnan(kp))
    bound = rotate_tol(f64(k), f64(gk), dtype, D).max() + half_step(dtype) * np.abs(np.nan_to_num(kp))
    assert (np.abs(np.nan_to_num(got) - np.nan_to_num(kp)) <= bound).all()
    assert written.sum() <= int(rowmask.sum()) * Hk * D
    tol = rotate_tol(f64(q), f64(gq), dtype, D) + half_step(dtype) * np.abs(qw)
    assert (np.abs(f64(qo) - qw)[rowmask] <= tol[rowmask]).all()
    assert (f64(qo)[~rowmask] == 5.0).all()                # rows behind the last sequence stay as they were
    assert int(c.status.item()) == 0

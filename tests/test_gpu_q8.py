"""The 8-bit paged cache (mrp_kv_append_q8, mrp_kv_read_q8, mrp_paged_attention_q8) and the attention of packed rows
(mrp_packed_attention, alone and joined) on the GPU against their 64-bit statements in oracle/kv.py.

Tolerances: those of test_gpu_kv.py on the values the cache holds (bf16 and f32 have all of them exactly), and
  append: a code is off by half a step, 2^-4 of the value or 2^-10 of the scale, from a row that is off by what the rotation is;
    values are not computed: their codes and scales are equal.
  join: log-sum-exps off by z (their own bounds) weigh the parts off by 2 z; the other pass's row carries its own rounding r."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import kv as ref
from test_gpu_kv import ATTEND, DEV, TORCH, U, Cache, f64, half_step, rotate_tol
from test_gpu_kv_paths import BIG, close, dense

gpu = pytest.mark.gpu


class CacheQ8(Cache):
    """A pool in 8 bits, with NaN rows wherever no position lies; k_pages and v_pages are the values it stands for."""

    def __init__(self, dtype, H, Hk, D, P, lens, seed=0, page_gap=0, **kw):
        super().__init__(dtype, H, Hk, D, P, lens, seed=seed, page_gap=page_gap, **kw)
        n_pages, self.gap = self.k_pages.shape[0], page_gap
        stride = Hk * P * D + page_gap
        self.codes, self.scales = [], []
        for pool in (self.k_pages, self.v_pages):
            rows = f64(pool)
            used = np.isfinite(rows).all(-1)
            size = np.exp(np.random.default_rng(seed + 7).standard_normal(rows.shape[:-1]))      # rows of different sizes
            codes, byte = ref.q8_rows(np.nan_to_num(rows) * size[..., None])
            junk = np.random.default_rng(seed).integers(0, 256, codes.shape, dtype=np.uint8)
            codes, byte = np.where(used[..., None], codes, junk), np.where(used, byte, 255).astype(np.uint8)
            c = torch.zeros(n_pages * stride, device=DEV, dtype=torch.uint8).as_strided((n_pages, Hk, P, D), (stride, P * D, D, 1))
            c.copy_(torch.from_numpy(codes).to(DEV))
            self.codes.append(c)
            self.scales.append(torch.from_numpy(byte).to(DEV))
        self.pool = self.b.KvPoolQ8(*self.codes, *self.scales)
        self.refresh()

    def refresh(self):
        """The values the pool stands for now."""
        self.k_pages, self.v_pages = (torch.from_numpy(ref.q8_values(c.cpu().numpy(), s.cpu().numpy())).to(DEV) for c, s in zip(self.codes, self.scales))

    def attend(self, q, out=None, lse=True, **kw):
        out = torch.full((q.shape[0], self.H, self.D), 7.0, device=DEV, dtype=q.dtype) if out is None else out
        lse = torch.full((q.shape[0], self.H), 7.0, device=DEV) if lse else None
        self.b.mrp_paged_attention_q8(self.ctx, self.batch, self.pool, q, out, lse, **kw)
        return out, lse

    def read(self, **kw):
        k, v = (torch.full((self.T, self.Hk, self.D), 7.0, device=DEV, dtype=TORCH[self.dtype]) for _ in range(2))
        self.b.mrp_kv_read_q8(self.ctx, self.batch, self.pool, k, v, **kw)
        return k, v


def name(c):
    return "%s-H%d-%d-D%d-P%d-n%d-m%d-w%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5]), c[6], c[7])


# ---- append, read ---------------------------------------------------------------------------------------------------

APPEND = [
    # dtype, H, Hk, D, P, lens, rot, interleaved, gap, norm
    ("bf16", 4, 2, 128, 16, [(0, 5), (15, 1), (16, 17), (3, 0), (40, 2)], 128, False, 0, True),
    ("bf16", 3, 1, 80, 7, [(6, 9), (0, 1)], 20, False, 64, True),
    ("bf16", 2, 2, 256, 32, [(31, 40)], 256, True, 0, False),
    ("f32", 4, 1, 64, 24, [(23, 2), (0, 30), (500, 1)], 48, False, 128, True),
    ("f32", 1, 1, 8, 1, [(2, 3)], 0, False, 0, False),
    ("f32", 3, 3, 72, 5, [(2, 13)], 36, False, 8, False),
    ("bf16", 8, 8, 64, 16, [(i, 1) for i in range(70)], 64, False, 0, True),
    ("bf16", 32, 8, 128, 64, [(100, 200), (0, 77)], 128, False, 0, True),
]


@gpu
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append_and_read(case):
    dtype, H, Hk, D, P, lens, rot, interleaved, gap, norm = case
    c = CacheQ8(dtype, H, Hk, D, P, lens, seed=1, rot=rot, interleaved=interleaved, extra_rows=3, page_gap=gap)
    rows = c.rand(c.T, H + 2 * Hk, D)
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    v *= torch.exp(c.rand(c.T, Hk, 1) * 3)
    gq, gk = (1 + 0.2 * c.rand(D), 1 + 0.2 * c.rand(D)) if norm else (None, None)
    before = [x.cpu().numpy().copy() for x in c.codes + c.scales]
    qo = torch.full((c.T, H, D), 5.0, device=DEV, dtype=TORCH[dtype])
    c.b.mrp_kv_append_q8(c.ctx, c.batch, c.pool, k, v, gk, q, qo, gq)
    ko, vo = c.read()
    pos, mine = np.zeros(c.T, np.int64), np.zeros(c.T, bool)
    for _, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * P):
        pos[s:s + n] = p + np.arange(n)
        mine[s:s + n] = True
    g64 = lambda t: None if t is None else f64(t)                              # noqa: E731
    kw, qw = (ref.norm_rotate(f64(x), pos, g64(gm), rot, 1e4, None, interleaved) for x, gm in ((k, gk), (q, gq)))
    codes, byte = ref.q8_rows(f64(v))
    after = [x.cpu().numpy() for x in c.codes + c.scales]
    want = [x.copy() for x in before]
    for b, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * P):
        for i in range(n):
            page, row = c.table_np[b, (p + i) // P], (p + i) % P
            want[1][page, :, row], want[3][page, :, row] = codes[s + i], byte[s + i]
            want[0][page, :, row], want[2][page, :, row] = after[0][page, :, row], after[2][page, :, row]
    for x, y in zip(after, want):                          # values exact, no other row touched
        assert np.array_equal(x, y)
    c.refresh()
    got = f64(ko)[mine]
    kscale = np.zeros((c.T, Hk))
    for b, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * P):
        for i in range(n):
            page, row = c.table_np[b, (p + i) // P], (p + i) % P
            kscale[s + i] = 2.0 ** (after[2][page, :, row].astype(np.float64) - 127)
            assert np.array_equal(f64(ko)[s + i], f64(c.k_pages)[page, :, row]) and np.array_equal(f64(vo)[s + i], f64(c.v_pages)[page, :, row])
    off = rotate_tol(f64(k), g64(gk), dtype, D)
    top = np.abs(kw).max(-1)
    assert (((top - off[..., 0]) <= 448 * kscale) & ((top + off[..., 0] > 224 * kscale) | (top == 0)))[mine].all()
    tol = off + np.maximum(np.abs(kw) * 2.0 ** -4, kscale[..., None] * 2.0 ** -10) * (1 + 2.0 ** -20)
    assert (np.abs(f64(ko) - kw) <= tol)[mine].all()
    assert (f64(ko)[~mine] == 7.0).all() and (f64(vo)[~mine] == 7.0).all() and (f64(qo)[~mine] == 5.0).all()
    assert got.size == 0 or np.isfinite(got).all()
    tol = rotate_tol(f64(q), g64(gq), dtype, D) + half_step(dtype) * np.abs(qw)
    assert (np.abs(f64(qo) - qw) <= tol)[mine].all()
    # the same queries as the append into a cache of the context type gives
    plain, other = torch.zeros((2,) + tuple(c.codes[0].shape), device=DEV, dtype=TORCH[dtype]), torch.full_like(qo, 5.0)
    if not gap:
        c.b.mrp_kv_append(c.ctx, c.batch, plain[0], plain[1], k, v, gk, q, other, gq)
        assert torch.equal(other, qo)
    # keys alone, values alone, strided rows
    wide = torch.full((c.T, 2 * Hk + 1, D), 7.0, device=DEV, dtype=TORCH[dtype])
    c.b.mrp_kv_read_q8(c.ctx, c.batch, c.pool, wide[:, 1:1 + Hk], None)
    assert torch.equal(wide[:, 1:1 + Hk], ko) and (wide[:, 0] == 7).all() and (wide[:, 1 + Hk:] == 7).all()
    c.b.mrp_kv_read_q8(c.ctx, c.batch, c.pool, None, wide[:, 1 + Hk:])
    assert torch.equal(wide[:, 1 + Hk:], vo)
    assert int(c.status.item()) == 0


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_not_finite_and_extreme_rows(dtype):
    """A row with NaN or infinity becomes a row of NaN, its neighbours stay; zeros, the largest and the smallest numbers."""
    c = CacheQ8(dtype, 2, 2, 64, 16, [(3, 20)], seed=2)
    k, v = c.rand(20, 2, 64), c.rand(20, 2, 64)
    big = torch.finfo(TORCH[dtype]).max
    for x in (k, v):
        x[1, 0, 5], x[2, 1, 63], x[3, 0, 0] = float("nan"), float("inf"), -float("inf")
        x[4, 1], x[5, 0], x[6] = 0.0, big, 2.0 ** -126
        x[7, 0], x[7, 1] = 2.0 ** -133, -0.0
        x[8] = 448.0
        x[9, :, :8] = torch.tensor([17.0, 18.0, 19.0, 21.0, 22.0, 23.0, 0.25, 448.0], device=DEV, dtype=TORCH[dtype])
    c.b.mrp_kv_append_q8(c.ctx, c.batch, c.pool, k, v)
    for x, codes, scales in ((k, c.codes[0], c.scales[0]), (v, c.codes[1], c.scales[1])):
        wc, ws = ref.q8_rows(f64(x))
        for i in range(20):
            page, row = c.table_np[0, (3 + i) // 16], (3 + i) % 16
            assert np.array_equal(scales[page, :, row].cpu().numpy(), ws[i]), i
            fine = ws[i] != 255
            assert np.array_equal(codes[page, :, row].cpu().numpy()[fine], wc[i][fine]), i
    ko, vo = c.read()
    for x, got in ((k, ko), (v, vo)):
        wc, ws = ref.q8_rows(f64(x))
        want = torch.from_numpy(ref.q8_values(wc, ws)).to(DEV).to(TORCH[dtype]).double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.double().nan_to_num(0.0), want.nan_to_num(0.0))
    c.codes[0][c.table_np[0, 0], 0, 3, 7] = 0x7F            # a code that append never writes reads as NaN
    assert torch.isnan(c.read()[0][0, 0, 7])


@gpu
@pytest.mark.parametrize("dtype,D,P,new", [("bf16", 128, 16, 2), ("bf16", 128, 16, 40), ("bf16", 128, 24, 300), ("bf16", 40, 9, 3), ("f32", 64, 16, 2)])
def test_sequences_and_pages_that_are_not_valid(dtype, D, P, new):
    lens = [(100, new), (60, new), (33, new), (200, new)]
    c = CacheQ8(dtype, 4, 2, D, P, lens, seed=3, extra_rows=5, rot=D)
    rows = c.rand(c.T, 8, D)
    q = rows[:, :4]
    good, lse = c.attend(q)
    c.check(q, good, lse)
    c.table_np[1, 1] = c.codes[0].shape[0] + 3
    c.table_np[2, 0] = -1
    c.table.copy_(torch.from_numpy(c.table_np))
    out, lse = c.attend(q)
    c.check(q, out, lse)
    assert int(c.status.item()) == c.b.MRP_DEV_BAD_INDEX
    assert c.b.mrp_fetch_status(c.ctx, clear=True) == c.b.MRP_DEV_BAD_INDEX

    def stored(reported=True):                             # (else: the pages of the new tokens are fine)
        before = [x.cpu().numpy().copy() for x in c.codes + c.scales]
        c.status.zero_()
        c.b.mrp_kv_append_q8(c.ctx, c.batch, c.pool, rows[:, 4:6], rows[:, 6:8], None, q, torch.empty_like(good))
        codes, byte = ref.q8_rows(f64(rows[:, 6:8]))
        for b, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * P):
            for i in range(n):
                page, row = c.table_np[b, (p + i) // P], (p + i) % P
                if 0 <= page < before[0].shape[0]:
                    before[1][page, :, row], before[3][page, :, row] = codes[s + i], byte[s + i]
                    before[0][page, :, row], before[2][page, :, row] = (x[page, :, row].cpu().numpy() for x in (c.codes[0], c.scales[0]))
        for x, y in zip(c.codes + c.scales, before):
            assert np.array_equal(x.cpu().numpy(), y)
        assert not reported or int(c.status.item()) & c.b.MRP_DEV_BAD_INDEX
        c.refresh()
        k, v = c.read()
        for b, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * P):
            want = ref.gather(f64(c.v_pages), c.table_np, b, p + n, P)[:, p:]
            assert np.array_equal(f64(v)[s:s + n], np.swapaxes(want, 0, 1))
    stored(False)
    for pre, start in (([-1, 60, 33, 200], None), ([100, 10 ** 9, 33, 200], None), ([2 ** 31 - 1, 60, 33, 200], None),
                       (None, [0, new, 2 * new, 3 * new, c.T + 9]), (None, [-4, new, 2 * new, 3 * new, 4 * new])):
        p0, s0 = c.pre_np, c.start_np
        c.pre_np = np.array(pre, np.int32) if pre else p0
        c.start_np = np.array(start, np.int32) if start else s0
        c.prefix_len.copy_(torch.from_numpy(c.pre_np))
        c.seq_start.copy_(torch.from_numpy(c.start_np))
        c.status.zero_()
        out, lse = c.attend(q)
        c.check(q, out, lse)
        assert int(c.status.item()) & c.b.MRP_DEV_BAD_INDEX
        stored()
        c.pre_np, c.start_np = p0, s0
        c.prefix_len.copy_(torch.from_numpy(p0))
        c.seq_start.copy_(torch.from_numpy(s0))


# ---- attention over pages in 8 bits -----------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("case", ATTEND, ids=name)
def test_attention_over_pages(case):
    dtype, H, Hk, D, P, lens, mask, window, sinks = case
    c = CacheQ8(dtype, H, Hk, D, P, lens, seed=H + D + P)
    q = c.rand(c.T, H, D) * 1.5
    kw = dict(mask=mask, window=window, sinks=sinks)
    out, lse = c.attend(q, **kw)
    c.check(q, out, lse, **kw)
    again, _ = c.attend(q, **kw)
    assert torch.equal(out, again)
    assert int(c.status.item()) == 0


@gpu
@pytest.mark.parametrize("case", BIG, ids=name)
def test_ragged_batches(case):
    dtype, H, Hk, D, P, lens, mask, window, sinks = case
    c = CacheQ8(dtype, H, Hk, D, P, lens, seed=D + len(lens))
    q = c.rand(c.T, H, D) * 1.5
    kw = dict(mask=mask, window=window, sinks=sinks)
    out, lse = c.attend(q, **kw)
    close(c, q, out, lse, **kw)
    for _ in range(4):
        again, lse2 = c.attend(q, **kw)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    for hint in (1, 10000):
        c.batch.c.max_new = hint
        o2, l2 = c.attend(q, **kw)
        close(c, q, o2, l2, **kw)
    assert int(c.status.item()) == 0
    assert c.b.mrp_fetch_status(c.ctx) == 0


# ---- rows over each other ---------------------------------------------------------------------------------------------

class Rows:
    """Sequences of packed rows; as a Cache whose pages are the rows of a sequence, for the checks on those."""

    def __init__(self, dtype, H, Hk, D, new, seed=0, extra_rows=0, flags=0, first=0):
        from paper_2605_18817_b200 import binding
        self.b, self.dtype, self.H, self.Hk, self.D = binding, dtype, H, Hk, D
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.rand = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=torch.float32).to(TORCH[dtype])
        self.start_np = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) + first
        self.T = int(self.start_np[-1]) + extra_rows
        rows = self.rand(self.T, H + 2 * Hk, D)
        self.q, self.k, self.v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
        self.q *= 1.5
        self.seq_start = torch.from_numpy(self.start_np).to(DEV)
        self.status = torch.zeros(1, device=DEV, dtype=torch.int32)
        self.ctx = binding.mrp_create(64, 64, 32, [], torch.zeros((32, 64), device=DEV, dtype=TORCH[dtype]), max_rows=1,
                                      max_seqs=max(1, len(new)), block_len=1, flags=flags)
        binding.mrp_kv_attach(self.ctx, H, Hk, D, 16)
        self.batch = binding.KvBatch(self.seq_start, None, None, self.T, max(list(new) + [0]), status=self.status)

    def attend(self, out=None, lse=True, **kw):
        out = torch.full((self.T, self.H, self.D), 7.0, device=DEV, dtype=TORCH[self.dtype]) if out is None else out
        lse = torch.full((self.T, self.H), 7.0, device=DEV) if lse is True else lse
        self.b.mrp_packed_attention(self.ctx, self.batch, self.k, self.v, self.q, out, lse if lse is not False else None, **kw)
        return out, lse

    def exact(self, mask=0, window=0, sinks=0, scale=0.0):
        """out, lse, reach, size in 64 bits on the device; rows of no sequence: 7."""
        g, scale = self.H // self.Hk, scale or 1 / math.sqrt(self.D)
        out, lse = torch.full((self.T, self.H, self.D), 7.0, dtype=torch.float64, device=DEV), torch.full((self.T, self.H), 7.0, dtype=torch.float64, device=DEV)
        reach, size, mine = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros(self.T, dtype=torch.bool, device=DEV)
        for b in range(len(self.start_np) - 1):
            s, e = int(self.start_np[b]), int(self.start_np[b + 1])
            if not 0 <= s <= e <= self.T or s == e:
                continue
            mine[s:e] = True
            x = self.q[s:e].double().transpose(0, 1)
            k, v = (y[s:e].double().transpose(0, 1).repeat_interleave(g, 0) for y in (self.k, self.v))
            i, j = torch.arange(e - s, device=DEV)[:, None], torch.arange(e - s, device=DEV)
            seen = (j <= i) if mask == 0 else torch.ones((e - s, e - s), dtype=torch.bool, device=DEV)
            if window:
                seen = seen & ((j > i - window) | (j < sinks))
            z = (x @ k.transpose(1, 2) * scale).masked_fill(~seen, -math.inf)
            w = torch.softmax(z, -1).nan_to_num(0.0)
            out[s:e], reach[s:e] = (w @ v).transpose(0, 1), (w @ v.abs()).transpose(0, 1)
            lse[s:e] = torch.logsumexp(z, -1).T
            size[s:e] = (x.abs() @ k.abs().transpose(1, 2) * scale).amax(-1).T
        return out, lse, reach, size, mine

    def score_error(self, size):
        return (self.D * U + (0.0 if self.dtype == "bf16" else 2.0 ** -20)) * size + 4 * U * (size + 1)

    def close(self, out, lse, rows=None, **kw):
        o, l, reach, size, mine = self.exact(**kw)
        n = int(np.diff(self.start_np).max()) + 1
        r, split = half_step(self.dtype), 0.0 if self.dtype == "bf16" else 2.0 ** -20
        z = self.score_error(size)
        tol = reach * (2 * z + 2 * n * U + (r if self.dtype == "bf16" else split))[..., None] + r * o.abs() + 1e-30
        ok = mine if rows is None else rows
        err = (out.double() - o).abs()
        assert torch.isfinite(out[ok].float()).all()
        assert (err[ok] <= tol[ok]).all(), (err / tol)[ok].max().item()
        assert (out[~mine] == 7.0).all()
        if lse is not False:
            assert (lse[~mine] == 7.0).all()
            empty = torch.isneginf(l)
            assert torch.equal(torch.isneginf(lse)[ok], empty[ok])
            fine = ok[:, None] & ~empty
            assert ((lse.double() - l).abs()[fine] <= (z + n * U + 4 * U * (l.abs() + 1))[fine]).all()


PACKED = [
    # dtype, H, Hk, D, new, mask, window, sinks
    ("bf16", 4, 2, 128, [1], 0, 0, 0),
    ("bf16", 4, 2, 128, [127, 128, 129, 1, 0, 2], 0, 0, 0),
    ("bf16", 4, 4, 64, [16] * 9, 1, 0, 0),
    ("bf16", 8, 1, 128, [300, 5, 64], 0, 0, 0),
    ("bf16", 8, 2, 128, [300, 700, 31], 0, 100, 7),
    ("bf16", 8, 2, 128, [300, 700, 31], 1, 100, 200),
    ("bf16", 16, 2, 128, [1000, 1], 0, 0, 0),
    ("bf16", 3, 1, 80, [50, 7, 130], 0, 0, 0),
    ("bf16", 5, 5, 8, [20, 13], 0, 0, 0),
    ("bf16", 4, 1, 200, [140, 33], 0, 1, 0),
    ("bf16", 4, 2, 256, [257, 3], 0, 0, 0),
    ("bf16", 2, 1, 64, [3] * 200, 1, 0, 0),
    ("bf16", 2, 1, 64, list(range(150)), 0, 0, 0),
    ("bf16", 32, 8, 128, [900, 1300, 2, 1], 0, 0, 0),                          # two row tiles a unit
    ("bf16", 32, 16, 64, [700] * 3 + [4] * 20, 0, 0, 0),
    ("bf16", 300, 2, 64, [70, 2], 0, 0, 0),
    ("f32", 4, 2, 64, [100, 1, 33], 0, 0, 0),
    ("f32", 6, 2, 40, [70, 8], 1, 9, 2),
    ("f32", 2, 2, 256, [40], 0, 0, 0),
    ("f32", 8, 2, 128, [77, 0, 20], 0, 30, 0),
]


@gpu
@pytest.mark.parametrize("case", PACKED, ids=lambda c: "%s-H%d-%d-D%d-n%d-m%d-w%d" % (c[0], c[1], c[2], c[3], len(c[4]), c[5], c[6]))
def test_packed_attention(case):
    dtype, H, Hk, D, new, mask, window, sinks = case
    c = Rows(dtype, H, Hk, D, new, seed=D + len(new), extra_rows=3)
    kw = dict(mask=mask, window=window, sinks=sinks)
    out, lse = c.attend(**kw)
    c.close(out, lse, **kw)
    for _ in range(4):
        again, l2 = c.attend(**kw)
        assert torch.equal(out, again) and torch.equal(lse, l2)
    for hint in (1, 10000):
        c.batch.c.max_new = hint
        o2, l2 = c.attend(**kw)
        c.close(o2, l2, **kw)
    assert torch.equal(c.attend(lse=False, **kw)[0], o2)
    assert int(c.status.item()) == 0 and c.b.mrp_fetch_status(c.ctx) == 0
    # on the tiles of 16 rows
    if dtype == "bf16":
        s = Rows(dtype, H, Hk, D, new, seed=D + len(new), extra_rows=3, flags=c.b.MRP_FLAG_FORCE_SIMT)
        s.close(*s.attend(**kw), **kw)


JOIN = [("bf16", 4, 2, 128, [4, 4, 4]), ("bf16", 32, 8, 128, [4] * 20), ("bf16", 8, 2, 128, [300, 1, 40]), ("bf16", 32, 8, 128, [900, 1300]),
        ("bf16", 5, 1, 80, [33, 2]), ("bf16", 4, 2, 256, [130, 3]), ("f32", 4, 2, 64, [4, 70, 1]), ("f32", 3, 3, 72, [9]), ("bf16", 300, 2, 64, [3, 2])]


@gpu
@pytest.mark.parametrize("case", JOIN, ids=str)
def test_joining_with_another_pass(case):
    dtype, H, Hk, D, new = case
    c = Rows(dtype, H, Hk, D, new, seed=5, extra_rows=2)
    o, l, reach, size, mine = c.exact(mask=1)
    prior, pl = c.rand(c.T, H, D), (c.rand(c.T, H).float() + l.float())
    pl[::3] = -math.inf                                     # saw nothing: its row is not read
    pl[1::7] += 40.0                                        # outweighs everything
    pl[2::7] -= 40.0
    prior[::3] = float("nan")
    out, lse = prior.clone(), pl.clone()
    out[~mine], lse[~mine] = 7.0, 7.0
    c.attend(out, lse, mask=1, join=True)
    want, lw = ref.join(f64(prior), f64(pl), f64(o), f64(l))
    n, r, split = max(new) + 1, half_step(dtype), 0.0 if dtype == "bf16" else 2.0 ** -20
    z = f64(c.score_error(size)) + n * U + 8 * U * (np.abs(f64(l)) + np.abs(np.where(np.isfinite(f64(pl)), f64(pl), 0.0)) + 2)
    mag = f64(reach) + np.abs(np.nan_to_num(f64(prior)))
    tol = mag * (2 * z[..., None] + 2 * n * U + (r if dtype == "bf16" else split)) + r * np.abs(want) + 1e-30
    m = f64(mine.float()) > 0
    assert np.isfinite(f64(out)[m]).all()
    assert (np.abs(f64(out) - want)[m] <= tol[m]).all(), (np.abs(f64(out) - want)[m] / tol[m]).max()
    assert (np.abs(f64(lse) - lw)[m] <= z[m] + 4 * U * (np.abs(lw[m]) + 1)).all()
    assert (out[~mine] == 7.0).all() and (lse[~mine] == 7.0).all()
    # nothing seen by either pass
    out, lse = torch.full_like(prior, float("nan")), torch.full_like(pl, -math.inf)
    keep = c.batch
    c.attend(out, lse, mask=1, join=True)
    alone, la = c.attend(mask=1)
    assert (out[mine].double() - alone[mine].double()).abs().max() <= 2 * r * alone[mine].double().abs().max() and torch.allclose(lse[mine], la[mine], atol=1e-5, rtol=0)
    assert keep is c.batch


@gpu
@pytest.mark.parametrize("dtype,new,pre", [("bf16", 4, 300), ("bf16", 32, 700), ("f32", 4, 100)])
def test_a_block_decoded_again_and_again(dtype, new, pre):
    """Prompts over themselves into the 8-bit cache, then blocks: over the cache in front of them joined with their own keys, twice,
    and stored once they are committed; against one 64-bit softmax over what the cache holds and the rows as they are."""
    H, Hk, D, P = 8, 2, 128, 16
    first = [pre, 1, pre // 2]
    total = [n + 2 * new for n in first]
    c = CacheQ8(dtype, H, Hk, D, P, [(0, t) for t in total], seed=2, rot=D, theta=1e4)
    gq, gk = 1 + 0.2 * c.rand(D), 1 + 0.2 * c.rand(D)
    done, r = [0, 0, 0], half_step(dtype)
    split = 0.0 if dtype == "bf16" else 2.0 ** -20
    for it in range(3):
        n = first if it == 0 else [new] * 3
        start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        batch = c.b.KvBatch(torch.from_numpy(start).to(DEV), torch.tensor(done, dtype=torch.int32, device=DEV), c.table, sum(n), max(n))
        for attempt in range(2 if it else 1):
            rows = c.rand(sum(n), H + 2 * Hk, D)
            q, k = (torch.empty((sum(n), h, D), device=DEV, dtype=TORCH[dtype]) for h in (H, Hk))
            out, lse = torch.empty_like(q), torch.empty((sum(n), H), device=DEV)
            pos = torch.cat([torch.arange(d, d + m, device=DEV, dtype=torch.int32) for d, m in zip(done, n)])
            c.b.mrp_qk_norm_rotate(c.ctx, pos, rows[:, :H], rows[:, H:H + Hk], q, k, gq, gk)
            v = rows[:, H + Hk:]
            if it == 0:
                c.b.mrp_packed_attention(c.ctx, batch, k, v, q, out, lse)
            else:
                c.b.mrp_paged_attention_q8(c.ctx, batch, c.pool, q, out, lse, mask=c.b.MRP_ATTN_PREFIX)
                c.b.mrp_packed_attention(c.ctx, batch, k, v, q, out, lse, mask=c.b.MRP_ATTN_BLOCK, join=True)
            c.refresh()
            for b in range(3):
                s, m, p = int(start[b]), n[b], done[b]
                pages = torch.from_numpy(c.table_np[b, :-(-p // P)].astype(np.int64)).to(DEV)
                held = [pool[pages].permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :p] for pool in (c.k_pages, c.v_pages)]
                kk, vv = (torch.cat([h, x[s:s + m].double().transpose(0, 1)], 1).repeat_interleave(H // Hk, 0) for h, x in zip(held, (k, v)))
                x = q[s:s + m].double().transpose(0, 1)
                seen = torch.ones((m, p + m), dtype=torch.bool, device=DEV)
                if it == 0:
                    seen = torch.arange(m, device=DEV)[:, None] >= torch.arange(m, device=DEV)
                zz = (x @ kk.transpose(1, 2) / math.sqrt(D)).masked_fill(~seen, -math.inf)
                w = torch.softmax(zz, -1)
                want, reach, lw = (w @ vv).transpose(0, 1), (w @ vv.abs()).transpose(0, 1), torch.logsumexp(zz, -1).T
                size = (x.abs() @ kk.abs().transpose(1, 2) / math.sqrt(D)).amax(-1).T
                z = (D * U + split) * size + 16 * U * (size + 2) + (p + m) * U
                # one rounding of the cache's part, one of the probabilities, one of the result
                tol = reach * (4 * z + (2 * r if dtype == "bf16" else 2 * split + r))[..., None] + r * want.abs()
                assert ((out[s:s + m].double() - want).abs() <= tol).all()
                assert ((lse[s:s + m].double() - lw).abs() <= 2 * z).all()
        c.b.mrp_kv_append_q8(c.ctx, batch, c.pool, rows[:, H:H + Hk], v, gk)
        done = [d + m for d, m in zip(done, n)]
    assert c.b.mrp_fetch_status(c.ctx) == 0


# ---- refusals ---------------------------------------------------------------------------------------------------------

@gpu
def test_refusals():
    c = CacheQ8("bf16", 4, 2, 128, 16, [(20, 3)], seed=1, rot=128)
    b, q = c.b, c.rand(3, 4, 128)
    out, k, v = torch.empty_like(q), c.rand(3, 2, 128), c.rand(3, 2, 128)
    lse = torch.empty((3, 4), device=DEV)

    def status(fn):
        with pytest.raises(b.MrpError) as e:
            fn()
        return e.value.status
    att = lambda **kw: b.mrp_paged_attention_q8(c.ctx, c.batch, c.pool, q, out, **kw)                    # noqa: E731
    pack = lambda k=k, v=v, q=q, out=out, lse=None, **kw: b.mrp_packed_attention(c.ctx, c.batch, k, v, q, out, lse, **kw)   # noqa: E731
    for kw in (dict(mask=3), dict(mask=-1), dict(window=-1), dict(sinks=-2), dict(scale=float("nan")), dict(scale=3e38), dict(scale=-1.0)):
        assert status(lambda: att(**kw)) == 1
        assert status(lambda: pack(**kw)) == 1
    assert status(lambda: pack(mask=b.MRP_ATTN_PREFIX)) == 1
    assert status(lambda: pack(join=True)) == 1             # nothing to join with
    assert status(lambda: pack(join=True, out=q, lse=lse)) == 1
    two = Rows("bf16", 2, 2, 128, [3])
    x = c.rand(3, 2, 128)
    assert status(lambda: b.mrp_packed_attention(two.ctx, two.batch, x, v, two.q, x, None)) == 1         # out is k
    fresh = b.mrp_create(64, 64, 32, [], torch.zeros((32, 64), device=DEV, dtype=torch.bfloat16), max_rows=1, max_seqs=1, block_len=1)
    for fn in (lambda: b.mrp_paged_attention_q8(fresh, c.batch, c.pool, q, out), lambda: b.mrp_packed_attention(fresh, c.batch, k, v, q, out),
               lambda: b.mrp_kv_append_q8(fresh, c.batch, c.pool, k, v), lambda: b.mrp_kv_read_q8(fresh, c.batch, c.pool, k, v)):
        assert status(fn) == 2
    b.mrp_kv_attach(fresh, 4, 2, 128, 16)                   # no cache: rows over each other alone
    b.mrp_packed_attention(fresh, b.KvBatch(c.seq_start, None, None, 3, 3), k, v, q, out)
    with pytest.raises(ValueError):
        b.mrp_paged_attention_q8(fresh, c.batch, c.pool, q, out)
    with pytest.raises(ValueError):
        b.mrp_paged_attention_q8(c.ctx, b.KvBatch(c.seq_start, None, None, 3, 3), c.pool, q, out)
    with pytest.raises(ValueError):
        b.KvBatch(c.seq_start, c.prefix_len, None, 3, 3)
    assert status(lambda: b.mrp_kv_read_q8(c.ctx, c.batch, c.pool, None, None)) == 1
    many = b.KvBatch(torch.zeros(3, dtype=torch.int32, device=DEV), None, None, 0, 0)
    assert status(lambda: b.mrp_packed_attention(c.ctx, many, k, v, q, out)) == 1                        # more than max_seqs
    for bad in (k.float(), k[:, :1], k[:2], k.transpose(0, 1), k.cpu()):
        for fn in (lambda: pack(k=bad), lambda: b.mrp_kv_append_q8(c.ctx, c.batch, c.pool, bad, v), lambda: b.mrp_kv_read_q8(c.ctx, c.batch, c.pool, k, bad)):
            with pytest.raises((TypeError, ValueError)):
                fn()
    kc, vc, ks, vs = c.codes + c.scales
    for bad in ((kc.int(), vc, ks, vs), (kc, vc[:-1], ks, vs), (kc, vc, ks.int(), vs), (kc, vc, ks, vs[:, :1]), (kc, vc, ks[:, :, ::2], vs), (kc.cpu(), vc, ks, vs)):
        with pytest.raises((TypeError, ValueError)):
            b.KvPoolQ8(*bad)
    odd = b.KvPoolQ8(kc.transpose(1, 2), vc.transpose(1, 2), ks.transpose(1, 2).contiguous(), vs.transpose(1, 2).contiguous())
    with pytest.raises(ValueError):
        b.mrp_paged_attention_q8(c.ctx, c.batch, odd, q, out)
    f8 = b.KvPoolQ8(kc.view(torch.float8_e4m3fn), vc.view(torch.float8_e4m3fn), ks.view(torch.float8_e8m0fnu), vs.view(torch.float8_e8m0fnu))
    b.mrp_paged_attention_q8(c.ctx, c.batch, f8, q, out, lse)
    c.check(q, out, lse)
    # unaligned pools and rows, overlapping rows
    a = b.mrp_attention_args(q.data_ptr(), out.data_ptr(), 512, 512, None, 0, 0, 0, 0.0)
    for i in range(4):
        p = b.mrp_kv_pool_q8(*(t.data_ptr() + (8 if i == j else 0) for j, t in enumerate((kc, vc, ks, vs))))
        assert b.lib.mrp_paged_attention_q8(c.ctx.handle, c.batch.ref, ctypes.byref(p), ctypes.byref(a), None) == 1
    store = torch.zeros(3 * 2 * 128 + 64, device=DEV, dtype=torch.bfloat16)
    assert status(lambda: pack(k=store[4:4 + 768].view(3, 2, 128))) == 1
    assert status(lambda: pack(v=store.as_strided((3, 2, 128), (248, 128, 1)))) == 1
    assert status(lambda: b.mrp_kv_read_q8(c.ctx, c.batch, c.pool, store.as_strided((3, 2, 128), (260, 128, 1)), v)) == 1
    out2, lse2 = c.attend(q)
    c.check(q, out2, lse2)


def test_refusals_on_the_host():
    from paper_2605_18817_b200 import binding as b
    for fn in (b.lib.mrp_kv_append_q8, b.lib.mrp_kv_read_q8, b.lib.mrp_paged_attention_q8, b.lib.mrp_packed_attention):
        assert fn(None, None, None, None, None) == 1
    with pytest.raises(TypeError):
        b.KvPoolQ8(*(torch.zeros((2, 1, 4, 8), dtype=torch.uint8) for _ in range(4)))


@gpu
@pytest.mark.parametrize("dtype,H,Hk,D,P,lens", [
    ("f32", 4, 2, 64, 16, [(30, 40), (5, 90)]), ("f32", 3, 1, 8, 1, [(2, 9)]), ("bf16", 3, 1, 80, 7, [(20, 33), (0, 40)]),
    ("bf16", 2, 2, 128, 8, [(64, 16), (32, 12)]), ("bf16", 4, 2, 128, 16, [(60, 32), (64, 64)]), ("bf16", 2, 2, 64, 32, [(90, 200), (0, 300)])],
    ids=str)
def test_the_cache_alone_needs_no_room_for_the_block(dtype, H, Hk, D, P, lens):
    c = CacheQ8(dtype, H, Hk, D, P, [(p, 0) for p, _ in lens], seed=D)
    cap = c.max_pages * P
    c.T = sum(n for _, n in lens)
    c.lens, c.start_np = lens, np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int32)
    c.seq_start = torch.from_numpy(c.start_np).to(DEV)
    c.batch = c.b.KvBatch(c.seq_start, c.prefix_len, c.table, c.T, max(n for _, n in lens), None, c.status)
    over = [p + n > cap for p, n in lens]
    q = c.rand(c.T, H, D)
    out, lse = c.attend(q, mask=c.b.MRP_ATTN_BLOCK)                # (elsewhere the rule stays)
    assert int(c.status) != 0 and any(over)
    c.status.zero_()
    for (p, n), s in zip(lens, c.start_np):
        assert p + n <= cap or bool((out[s:s + n] == 7).all() and (lse[s:s + n] == 7).all())
    c.max_pages = 1 << 20                                          # what the plain form refuses by
    for window in (0, 50):
        out, lse = c.attend(q, mask=c.b.MRP_ATTN_PREFIX, window=window)
        close(c, q, out, lse, mask=2, window=window)
    assert int(c.status) == 0

"""The 8-bit cache and packed attention where they can go wrong: captured and replayed calls, other streams, offsets beyond 32
bits, rows that are not finite or at the end of the types' range in places that some do not see, maxima that grow from tile to tile,
long tails, outputs in place, empty batches.  Tolerances as in test_gpu_q8.py."""
import math

import numpy as np
import pytest
import torch

from oracle import kv as ref
from test_gpu_kv import DEV, TORCH, U, f64, half_step
from test_gpu_kv_paths import close, dense
from test_gpu_kv_rising import RISING
from test_gpu_kv_values import VALUES, check_lse
from test_gpu_q8 import CacheQ8, Rows

gpu = pytest.mark.gpu
LOG2E = 1.4426950408889634


def put_row(c, which, pos, values, seq=0):
    """Position `pos` of a sequence: the keys (0) or values (1) of all heads become `values` [Hk, D], quantised."""
    codes, byte = ref.q8_rows(np.broadcast_to(np.asarray(values, np.float64), (c.Hk, c.D)))
    page, row = c.table_np[seq, pos // c.P], pos % c.P
    c.codes[which][page, :, row], c.scales[which][page, :, row] = torch.from_numpy(codes).to(DEV), torch.from_numpy(byte).to(DEV)
    c.refresh()


def kept(c):
    return [x.clone() for x in c.codes + c.scales]


def put_back(c, saved):
    for x, y in zip(c.codes + c.scales, saved):
        x.copy_(y)
    c.refresh()


@gpu
@pytest.mark.parametrize("where", ["some rows", "all rows"])
@pytest.mark.parametrize("case", VALUES, ids=lambda c: "%s-H%d-%d-D%d-P%d-n%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5])))
def test_rows_of_nan_reach_only_the_rows_that_see_them(case, where):
    dtype, H, Hk, D, P, lens, at = case
    c = CacheQ8(dtype, H, Hk, D, P, lens, seed=D)
    q = c.rand(c.T, H, D)
    if where == "all rows":
        at = lens[0][0] // 2
    saved = kept(c)
    clean = torch.ones(c.T, dtype=torch.bool, device=DEV)
    clean[max(0, at - lens[0][0]):lens[0][1]] = False
    before = (c.k_pages, c.v_pages)
    for which in (1, 0):
        put_row(c, which, at, np.nan)
        out, lse = c.attend(q)
        assert torch.isnan(out[~clean].float()).all()
        put_back(c, saved)
        if which == 1:
            check_lse(c, q, lse)                           # a log-sum-exp knows nothing of values
        else:
            assert torch.isnan(lse[~clean]).all()
        close(c, q, out, lse, rows=clean)
    assert all(torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0)) for a, b in zip(before, (c.k_pages, c.v_pages)))


@gpu
@pytest.mark.parametrize("dtype,D,P,new", [("f32", 64, 16, 9), ("f32", 128, 24, 30), ("bf16", 64, 20, 9), ("bf16", 128, 16, 3), ("bf16", 128, 16, 7),
                                           ("bf16", 256, 16, 3), ("bf16", 128, 16, 40), ("bf16", 64, 32, 40), ("bf16", 128, 32, 300)])
def test_extreme_rows_reach_only_the_rows_that_see_them(dtype, D, P, new):
    c = CacheQ8(dtype, 4, 2, D, P, [(150, new), (40, new)], seed=D)
    q = c.rand(c.T, 4, D)
    at = 150 + new // 2
    clean = torch.ones(c.T, dtype=torch.bool, device=DEV)
    clean[new // 2:new] = False
    saved = kept(c)
    for what in (torch.finfo(q.dtype).max, torch.finfo(q.dtype).min):
        for which in (1, 0):
            put_row(c, which, at, what)
            out, lse = c.attend(q)
            if which == 1:
                check_lse(c, q, lse)
            put_back(c, saved)
            close(c, q, out, lse, rows=clean)


@gpu
@pytest.mark.parametrize("D,P,new", [(128, 16, 1), (128, 16, 4), (256, 16, 2), (128, 16, 40), (64, 32, 40), (128, 64, 300), (80, 24, 3)])
def test_rows_of_very_different_sizes(D, P, new):
    """Scales from 2^-127 to 2^100, rows of zeros among them: V's factors in one or two products, K's in the score."""
    c = CacheQ8("bf16", 4, 2, D, P, [(300, new), (77, new)], seed=3)
    rng = np.random.default_rng(1)
    for b, (p, n) in enumerate(c.lens):
        for j in range(p + n):
            row = rng.standard_normal((2, D))
            if j % 7 == 0:
                put = row * 2.0 ** rng.integers(-60, -8)
            elif j % 7 == 1:
                put = row * 0.0
            elif j % 7 == 2:
                put = row * 2.0 ** rng.integers(9, 90)
            elif j == 33:
                put = row * 2.0 ** -130
            else:
                continue
            codes, byte = ref.q8_rows(put)
            page, r = c.table_np[b, j // P], j % P
            c.codes[1][page, :, r], c.scales[1][page, :, r] = torch.from_numpy(codes).to(DEV), torch.from_numpy(byte).to(DEV)
            if j % 7 < 2:                                  # (keys of huge scores would leave one position alone)
                c.codes[0][page, :, r], c.scales[0][page, :, r] = torch.from_numpy(codes).to(DEV), torch.from_numpy(byte).to(DEV)
    c.refresh()
    q = c.rand(c.T, 4, D)
    out, lse = c.attend(q)
    close(c, q, out, lse)


@gpu
@pytest.mark.parametrize("new", [1, 4, 30])
def test_queries_of_any_size(new):
    """Rows from 2^-100 to 2^60 with keys to match, elements 2^-20 of their row's largest, rows of zeros, and rows that are not
    finite, which stay with themselves.  Up to 16 rows go as two e4m3 parts: to 2^-21 of the row's largest element."""
    c = CacheQ8("bf16", 4, 2, 128, 16, [(200, new), (50, new)], seed=4)
    q = c.rand(c.T, 4, 128)
    q[0, 0] *= 2.0 ** -100
    q[0, 1] = 0.0
    q[-1, 2, ::2] *= 2.0 ** -20
    q[-1, 3, 1:] *= 2.0 ** -13
    out, lse = c.attend(q)
    o, l, reach, size = dense(c, q)
    extra = torch.zeros_like(size)
    for b, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * 16):
        pages = torch.from_numpy(c.table_np[b, :-(-(p + n) // 16)].astype(np.int64)).to(DEV)
        k = c.k_pages[pages].permute(1, 0, 2, 3).reshape(2, -1, 128)[:, :p + n].repeat_interleave(2, 0)
        extra[s:s + n] = 2.0 ** -21 * q[s:s + n].double().abs().amax(-1) * k.abs().sum(-1).amax(-1) / math.sqrt(128)
    z = 128 * U * size + 4 * U * (size + 1) + extra
    assert ((out.double() - o).abs() <= reach * (2 * z + 600 * U + 2.0 ** -8)[..., None] + 2.0 ** -8 * o.abs()).all()
    assert ((lse.double() - l).abs() <= z + 300 * U + 4 * U * (l.abs() + 1)).all()
    good = out.clone()
    for what in (float("nan"), float("inf")):
        q2 = q.clone()
        q2[0, 2, 5] = what
        out, lse = c.attend(q2)
        assert torch.isnan(out[0, 2].float()).all() and torch.isnan(lse[0, 2])
        out[0, 2] = good[0, 2]
        assert torch.equal(out, good)


@gpu
@pytest.mark.parametrize("rows", ["all", "some"])
@pytest.mark.parametrize("case", RISING, ids=lambda c: "%s-H%d-%d-D%d-P%d-n%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5])))
def test_scores_that_rise_along_the_cache(case, rows):
    dtype, H, Hk, D, P, lens, mask = case
    c = CacheQ8(dtype, H, Hk, D, P, lens, seed=D)
    k = c.k_pages.cpu().numpy()
    for b, (p, n) in enumerate(lens):                      # feature 0 of a key: the height of its tile
        for j in range(p + n):
            page, row = c.table_np[b, j // P], j % P
            k[page, :, row, 0] = (j // 128) * (3.0 * math.sqrt(D) / LOG2E)
    used = np.isfinite(k).all(-1)
    codes, byte = ref.q8_rows(np.nan_to_num(k))
    c.codes[0].copy_(torch.from_numpy(np.where(used[..., None], codes, c.codes[0].cpu().numpy())).to(DEV))
    c.scales[0].copy_(torch.from_numpy(np.where(used, byte, 255).astype(np.uint8)).to(DEV))
    c.refresh()
    q = c.rand(c.T, H, D)
    parts = torch.tensor([1.0] if rows == "all" else [1.0, 0.0, -1.0, 0.5], device=DEV)
    q[..., 0] = parts[(torch.arange(c.T, device=DEV)[:, None] + torch.arange(H, device=DEV)) % len(parts)].to(q.dtype)
    out, lse = c.attend(q, mask=mask)
    close(c, q, out, lse, mask=mask)


@gpu
@pytest.mark.parametrize("new,H", [(1, 4), (4, 8), (20, 8)])
def test_a_long_tail_behind_one_large_probability(new, H):
    """One position far above 60000 others, which together weigh as much: none of them is lost."""
    n = 60000
    c = CacheQ8("bf16", H, 2, 128, 64, [(n, new)], seed=6)
    c.codes[0].zero_()
    c.scales[0].fill_(127)
    q = torch.zeros((new, H, 128), device=DEV, dtype=torch.bfloat16)
    q[..., 0] = 1.0
    put_row(c, 0, 123, np.eye(1, 128)[0] * 120.0)          # score 120 / sqrt(128) = 10.6: e^10.6 is two thirds of the others' sum
    out, lse = c.attend(q)
    close(c, q, out, lse)


@gpu
@pytest.mark.parametrize("dtype,D,new", [("bf16", 128, 1), ("bf16", 128, 4), ("bf16", 128, 24), ("bf16", 64, 150), ("f32", 64, 3)])
def test_a_captured_step_serves_other_lengths(dtype, D, new):
    """Append, attention over the cache, join with the block's own rows, reading back: captured once, replayed with other lengths
    and contents, against the same calls made directly (which are held to 64 bits elsewhere)."""
    lens = [(700, new), (64, new), (300, new)]
    c = CacheQ8(dtype, 4, 2, D, 16, lens, seed=8, rot=D)
    rows = c.rand(c.T, 8, D)
    dt = TORCH[dtype]
    q, out, ko, vo = (torch.empty((c.T, h, D), device=DEV, dtype=dt) for h in (4, 4, 2, 2))
    lse, l2, out2 = torch.empty((c.T, 4), device=DEV), torch.empty((c.T, 4), device=DEV), torch.empty_like(out)

    def step():
        c.b.mrp_kv_append_q8(c.ctx, c.batch, c.pool, rows[:, 4:6], rows[:, 6:8], None, rows[:, :4], q)
        c.b.mrp_paged_attention_q8(c.ctx, c.batch, c.pool, q, out, lse)
        c.b.mrp_kv_read_q8(c.ctx, c.batch, c.pool, ko, vo)
        c.b.mrp_paged_attention_q8(c.ctx, c.batch, c.pool, q, out2, l2, mask=c.b.MRP_ATTN_PREFIX)
        c.b.mrp_packed_attention(c.ctx, c.batch, ko, vo, q, out2, l2, join=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for pre in ([700, 64, 300], [1, 0, 250], [699, 17, 5]):
        c.pre_np = np.array(pre, np.int32)
        c.prefix_len.copy_(torch.from_numpy(c.pre_np))
        rows.copy_(c.rand(c.T, 8, D))
        saved = kept(c)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, ko, vo, out2, l2, *c.codes, *c.scales)]
        put_back(c, saved)
        for x in (out, lse, ko, vo, out2, l2):
            x.fill_(7.0)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, ko, vo, out2, l2, *c.codes, *c.scales)))
        c.refresh()
        c.lens = [(p, new) for p in pre]
        close(c, q, out, lse)
        # the joined passes see the same positions (the block's rows as the cache holds them): twice rounded
        r = half_step(dtype)
        assert ((out2.double() - out.double()).abs() <= 4 * r * (out.double().abs() + dense(c, q)[2]) + 1e-5).all()
        assert ((l2 - lse).abs() <= 1e-4).all()
    assert int(c.status.item()) == 0


@gpu
def test_two_contexts_on_two_streams_at_once():
    cs = [CacheQ8("bf16", 32, 8, 128, 16, [(1500, n), (900, n), (30, n)], seed=n) for n in (1, 4, 40)]
    qs = [c.rand(c.T, 32, 128) for c in cs]
    ps = [Rows("bf16", 32, 8, 128, [n] * 5, seed=n) for n in (4, 200)]
    want, wantp = [c.attend(q) for c, q in zip(cs, qs)], [p.attend(mask=1) for p in ps]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(5)], []
    for _ in range(20):
        for i, (c, q) in enumerate(zip(cs, qs)):
            out, lse = torch.full_like(want[i][0], 7.0), torch.full_like(want[i][1], 7.0)
            streams[i].wait_stream(torch.cuda.current_stream())
            c.b.mrp_paged_attention_q8(c.ctx, c.batch, c.pool, q, out, lse, stream=streams[i])
            got.append((want[i], out, lse))
        for i, p in enumerate(ps):
            out, lse = torch.full_like(wantp[i][0], 7.0), torch.full_like(wantp[i][1], 7.0)
            streams[3 + i].wait_stream(torch.cuda.current_stream())
            p.b.mrp_packed_attention(p.ctx, p.batch, p.k, p.v, p.q, out, lse, mask=1, stream=streams[3 + i])
            got.append((wantp[i], out, lse))
    torch.cuda.synchronize()
    for w, out, lse in got:
        assert torch.equal(out, w[0]) and torch.equal(lse, w[1])


@gpu
@pytest.mark.parametrize("new", [1, 4, 30])
@pytest.mark.parametrize("P,D", [(16, 128), (20, 128)])
def test_offsets_beyond_32_bits(new, P, D):
    """Pages so far apart that the last ones lie 2^32 bytes on: a pool of which little is touched."""
    lens = [(3 * P - 1, new)]
    c = CacheQ8("bf16", 4, 2, D, P, lens, seed=4, spare_pages=0, rot=D)
    n_pages, page = c.codes[0].shape[0], 2 * P * D
    stride = (2 ** 32 + 4096) // max(1, n_pages - 2)
    stride -= stride % 16
    c.b.mrp_kv_attach(c.ctx, 4, 2, D, P, n_pages, c.max_pages, stride, D)
    pools = []
    for pool in c.codes:
        big = torch.empty((n_pages - 1) * stride + page, device=DEV, dtype=torch.uint8).as_strided((n_pages, 2, P, D), (stride, P * D, D, 1))
        big.copy_(pool)
        pools.append(big)
    assert (n_pages - 1) * stride > 2 ** 32
    c.codes, c.pool = pools, c.b.KvPoolQ8(*pools, *c.scales)
    rows = c.rand(c.T, 8, D)
    q = torch.empty((c.T, 4, D), device=DEV, dtype=torch.bfloat16)
    c.b.mrp_kv_append_q8(c.ctx, c.batch, c.pool, rows[:, 4:6], rows[:, 6:8], None, rows[:, :4], q)
    c.refresh()
    out, lse = c.attend(q)
    c.check(q, out, lse)
    codes, byte = ref.q8_rows(f64(rows[:, 6:8]))
    _, v = c.read()
    assert np.array_equal(f64(v), ref.q8_values(codes, byte))


@gpu
@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 4), ("bf16", 20), ("bf16", 150), ("f32", 3)])
def test_attention_in_place(dtype, new):
    c = CacheQ8(dtype, 8, 2, 128, 16, [(3000, new), (70, new), (0, new)], seed=5)
    q = c.rand(c.T, 8, 128)
    out, lse = c.attend(q)
    c.check(q, out, lse)
    same = q.clone()
    again, l2 = c.attend(same, same)
    assert torch.equal(again, out) and torch.equal(l2, lse)
    p = Rows(dtype, 8, 2, 128, [new, 3, new], seed=5)
    out, lse = p.attend()
    p.close(out, lse)
    p.q = p.q.contiguous()
    l2 = torch.empty_like(lse)
    p.b.mrp_packed_attention(p.ctx, p.batch, p.k, p.v, p.q, p.q, l2)
    assert torch.equal(p.q, out) and torch.equal(l2, lse)


@gpu
@pytest.mark.parametrize("gap", [16, 8, 1024])
@pytest.mark.parametrize("D,P,new", [(128, 16, 1), (128, 24, 9), (128, 32, 40), (256, 8, 2), (72, 16, 3), (128, 16, 200), (16, 8, 5)])
def test_small_pages_with_gaps(D, P, new, gap):
    c = CacheQ8("bf16", 4, 2, D, P, [(500, new), (P - 1, new), (1, new)], seed=7, page_gap=gap)
    q = c.rand(c.T, 4, D)
    out, lse = c.attend(q)
    c.check(q, out, lse)


@gpu
@pytest.mark.parametrize("D,new", [(128, 5), (128, 90), (64, 300), (256, 20), (80, 33)])
def test_values_that_are_not_finite_in_packed_rows(D, new):
    for what in (float("nan"), float("inf"), torch.finfo(torch.bfloat16).max):
        c = Rows("bf16", 4, 2, D, [new, new, 1], seed=5)
        at = new // 2
        good = c.v[at].clone()
        c.v[at] = what
        out, lse = c.attend()
        clean = torch.ones(c.T, dtype=torch.bool, device=DEV)
        clean[at:new] = False
        assert 1e38 < what < float("inf") or not torch.isfinite(out[at:new].float()).any()
        c.v[at] = good
        c.close(out, lse, rows=clean)
        c.close(c.attend()[0], lse)                        # log-sum-exps know nothing of values
        good = c.k[at].clone()
        c.k[at] = what
        out, lse = c.attend()
        c.k[at] = good
        c.close(out, lse, rows=clean)
        if new <= 90:                                      # what lies behind the last sequence reaches nobody
            c = Rows("bf16", 4, 2, D, [new, 3], seed=6, extra_rows=40)
            want = c.attend(mask=1)
            c.k[-40:], c.v[-40:] = what, what
            got = c.attend(mask=1)
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@gpu
@pytest.mark.parametrize("new", [4, 200])
def test_packed_rows_and_sequences_that_do_not_fit(new):
    c = Rows("bf16", 4, 2, 128, [new] * 4, seed=9, extra_rows=5)
    for start in ([0, 10 * new, 2 * new, 3 * new, 4 * new], [-3, new, 2 * new, 3 * new, 4 * new], [0, new, 2 * new, 2 * new - 1, c.T + 1]):
        c.start_np = np.array(start, np.int32)
        c.seq_start.copy_(torch.from_numpy(c.start_np))
        c.status.zero_()
        out, lse = c.attend()
        c.close(out, lse)
        assert int(c.status.item()) == c.b.MRP_DEV_BAD_INDEX
    assert c.b.mrp_fetch_status(c.ctx, clear=True) == c.b.MRP_DEV_BAD_INDEX
    # a cached batch serves too: its prefix and pages are not read
    c.seq_start.copy_(torch.arange(0, 4 * new + 1, new, dtype=torch.int32, device=DEV))
    c.start_np = np.arange(0, 4 * new + 1, new).astype(np.int32)
    want = c.attend()
    junk = torch.full((4,), -5, dtype=torch.int32, device=DEV)
    c.batch = c.b.KvBatch(c.seq_start, junk, junk[:, None].contiguous(), c.T, new, status=c.status)
    c.status.zero_()
    got = c.attend()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and int(c.status.item()) == 0


@gpu
def test_empty_batches_and_empty_sequences():
    c = CacheQ8("bf16", 4, 2, 128, 16, [(20, 0), (30, 3), (0, 0)], seed=1)
    q = c.rand(c.T, 4, 128)
    out, lse = c.attend(q)
    c.check(q, out, lse)
    none = c.b.KvBatch(c.seq_start[:1], c.prefix_len[:0], c.table[:0], 0, 0)
    out = torch.full((3, 4, 128), 7.0, device=DEV, dtype=torch.bfloat16)
    k = q[:, :2]
    c.b.mrp_paged_attention_q8(c.ctx, none, c.pool, q, out)
    c.b.mrp_kv_append_q8(c.ctx, none, c.pool, k, k)
    c.b.mrp_kv_read_q8(c.ctx, none, c.pool, out[:, :2], None)
    c.b.mrp_packed_attention(c.ctx, none, k, k, q, out)
    assert c.ctx.last_launch_count == 0
    zeros = torch.zeros(2, dtype=torch.int32, device=DEV)  # sequences, but not a token among them
    b = c.b.KvBatch(zeros, zeros[:1], c.table[:1], 3, 1)
    c.b.mrp_paged_attention_q8(c.ctx, b, c.pool, q, out)
    c.b.mrp_kv_read_q8(c.ctx, b, c.pool, out[:, :2], None)
    c.b.mrp_packed_attention(c.ctx, b, k, k, q, out)
    b.c.max_new = 500
    c.b.mrp_paged_attention_q8(c.ctx, b, c.pool, q, out)
    c.b.mrp_packed_attention(c.ctx, b, k, k, q, out)
    torch.cuda.synchronize()
    assert (out == 7).all()


@gpu
def test_the_kernels_of_a_geometry_agree():
    lens = [(333, 40), (900, 2), (0, 129), (50, 4)]
    c = CacheQ8("bf16", 8, 2, 128, 32, lens, seed=12)
    q = c.rand(c.T, 8, 128)
    out, lse = c.attend(q)
    other = c.b.mrp_create(64, 64, 32, [], torch.zeros((32, 64), device=DEV, dtype=torch.bfloat16), max_rows=1, max_seqs=4, block_len=1,
                           flags=c.b.MRP_FLAG_FORCE_SIMT)
    c.b.mrp_kv_attach(other, 8, 2, 128, 32, c.codes[0].shape[0], c.max_pages)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    c.b.mrp_paged_attention_q8(other, c.batch, c.pool, q, o2, l2)
    close(c, q, o2, l2)
    close(c, q, out, lse)
    assert (lse - l2).abs().max() < 1e-4

"""The paged-cache operators where they can go wrong: every kernel over ragged batches, values that are not finite in
places that are not seen, indices that are not valid, captured and replayed calls, other streams, strides and offsets
beyond 32 bits, refusals, and a run of all of them as a decoding loop uses them.  Tolerances as in test_gpu_kv.py."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import kv as ref
from test_gpu_kv import DEV, TORCH, U, Cache, f64, half_step

gpu = pytest.mark.gpu


def dense(c, q, mask=0, window=0, sinks=0):
    """The statement of oracle/kv.py, sequence by sequence in 64 bits on the device: out, lse, reach, size."""
    T, g = q.shape[0], c.H // c.Hk
    out, reach = (torch.zeros(q.shape, dtype=torch.float64, device=DEV) for _ in range(2))
    lse, size = (torch.zeros(T, c.H, dtype=torch.float64, device=DEV) for _ in range(2))
    for b, s, n, p in ref.sequences(c.start_np, c.pre_np, T, c.max_pages * c.P):
        length = p if mask == 2 else p + n
        if n == 0:
            continue
        pages = torch.from_numpy(c.table_np[b, :-(-length // c.P)].astype(np.int64)).to(DEV)
        k, v = (pool[pages].double().permute(1, 0, 2, 3).reshape(c.Hk, -1, c.D)[:, :length].repeat_interleave(g, 0) for pool in (c.k_pages, c.v_pages))
        pos, j = p + torch.arange(n, device=DEV)[:, None], torch.arange(length, device=DEV)
        seen = (j <= pos) if mask == 0 else torch.ones((n, length), dtype=torch.bool, device=DEV)
        if window:
            seen = seen & ((j > pos - window) | (j < sinks))
        x = q[s:s + n].double().transpose(0, 1)
        z = (torch.einsum("hnd,hjd->hnj", x, k) / math.sqrt(c.D)).masked_fill(~seen, -math.inf)
        w = torch.softmax(z, -1).nan_to_num(0.0)
        out[s:s + n], reach[s:s + n] = (torch.einsum("hnj,hjd->nhd", w, y) for y in (v, v.abs()))
        lse[s:s + n] = torch.logsumexp(z, -1).T if length else -math.inf
        if length:
            size[s:s + n] = (torch.einsum("hnd,hjd->hnj", x.abs(), k.abs()) / math.sqrt(c.D)).amax(-1).T
    return out, lse, reach, size


def close(c, q, out, lse, mask=0, window=0, sinks=0, rows=None):
    o, l, reach, size = dense(c, q, mask, window, sinks)
    n = max(p + m for p, m in c.lens) + 1
    r, split = half_step(c.dtype), 0.0 if c.dtype == "bf16" else 2.0 ** -20
    z = (c.D * U + split) * size + 4 * U * (size + 1)
    tol = reach * (2 * z + 2 * n * U + (r if c.dtype == "bf16" else split))[..., None] + r * o.abs() + 1e-30
    err = (out.double() - o).abs()
    ok = torch.ones(q.shape[0], dtype=torch.bool, device=DEV) if rows is None else rows
    assert torch.isfinite(out[ok].float()).all()
    assert (err[ok] <= tol[ok]).all(), (err / tol)[ok].max().item()
    empty = torch.isneginf(l)
    assert torch.equal(torch.isneginf(lse)[ok], empty[ok])
    fine = ok[:, None] & ~empty
    lt = z + n * U + 4 * U * (l.abs() + 1)
    assert ((lse.double() - l).abs()[fine] <= lt[fine]).all()


BIG = [
    # dtype, H, Hk, D, P, lens, mask, window, sinks
    ("bf16", 32, 8, 128, 64, [(37 * i % 3000, 1) for i in range(40)], 0, 0, 0),              # single tokens, many units a CTA
    ("bf16", 32, 8, 128, 32, [(61 * i % 2500, 16) for i in range(1, 13)], 1, 0, 0),          # blocks of 16
    ("bf16", 16, 8, 64, 16, [(97 * i % 900, 1 + 13 * i % 31) for i in range(30)], 0, 0, 0),
    ("bf16", 8, 2, 128, 128, [(5000, 1), (100, 700), (0, 333), (2000, 129)], 0, 0, 0),       # prompts
    ("bf16", 8, 2, 128, 16, [(900, 1)] * 30 + [(500, 400)], 0, 0, 0),                        # single tokens beside a prompt
    ("bf16", 6, 2, 80, 24, [(700, 1)] * 9 + [(3, 130), (64, 43)], 0, 0, 0),
    ("bf16", 16, 1, 128, 64, [(2000, 9), (40, 200)], 0, 300, 70),                            # window over many rows
    ("bf16", 16, 1, 128, 64, [(2000, 9), (40, 200), (0, 130)], 2, 60, 0),                    # most rows see nothing
    ("bf16", 4, 4, 96, 40, [(333, 140), (129, 128), (127, 1)], 1, 128, 128),
    ("bf16", 4, 2, 128, 32, [(20 + i, 20) for i in range(140)], 0, 0, 0),                    # more than 128 sequences
    ("bf16", 4, 2, 128, 32, [(130 + i, 1) for i in range(300)], 0, 0, 0),
    ("bf16", 4, 2, 72, 100, [(1000, 30), (77, 1)], 0, 0, 0),                                 # pages that TMA boxes do not tile
    ("bf16", 8, 1, 256, 32, [(1500, 2), (300, 70)], 0, 0, 0),
    ("bf16", 16, 4, 256, 16, [(37 * i % 1500, 1) for i in range(40)], 0, 0, 0),
    ("bf16", 8, 2, 200, 16, [(1000, 4), (333, 1), (0, 4)], 1, 0, 0),
    ("bf16", 8, 2, 136, 64, [(700, 150), (129, 33), (0, 260)], 0, 100, 7),
    ("bf16", 12, 4, 40, 16, [(900, 1), (131, 5), (0, 3)], 0, 0, 0),
    ("bf16", 12, 4, 24, 32, [(700, 40), (0, 130)], 0, 0, 0),
    ("bf16", 6, 1, 8, 8, [(500, 2), (77, 30)], 0, 0, 0),
    ("f32", 8, 2, 128, 16, [(1200, 1), (700, 30), (0, 90)], 0, 0, 0),
    ("bf16", 300, 1, 64, 16, [(140, 2), (0, 1), (700, 1)], 0, 0, 0),                         # a token's heads over several row tiles
    ("bf16", 300, 2, 128, 32, [(140, 5), (0, 1)], 0, 64, 4),
    ("f32", 50, 1, 32, 16, [(140, 2), (0, 1)], 0, 0, 0),
]


@gpu
@pytest.mark.parametrize("case", BIG, ids=lambda c: "%s-H%d-%d-D%d-P%d-n%d-m%d-w%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5]), c[6], c[7]))
def test_ragged_batches(case):
    dtype, H, Hk, D, P, lens, mask, window, sinks = case
    c = Cache(dtype, H, Hk, D, P, lens, seed=D + len(lens))
    q = c.rand(c.T, H, D) * 1.5
    kw = dict(mask=mask, window=window, sinks=sinks)
    out, lse = c.attend(q, **kw)
    close(c, q, out, lse, **kw)
    for _ in range(8):
        again, lse2 = c.attend(q, **kw)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    # what the host believes of the longest block chooses kernels, never results beyond rounding
    for hint in (1, 10000):
        c.batch.c.max_new = hint
        o2, l2 = c.attend(q, **kw)
        close(c, q, o2, l2, **kw)
    assert int(c.status.item()) == 0
    assert c.b.mrp_fetch_status(c.ctx) == 0


@gpu
@pytest.mark.parametrize("D,P,new", [(128, 16, 3), (128, 16, 20), (128, 64, 200), (64, 32, 40), (80, 7, 30), (256, 16, 12)])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(D, P, new):
    c = Cache("bf16", 4, 2, D, P, [(150, new), (40, new)], seed=5)
    q = c.rand(c.T, 4, D)
    bad = 150 + new // 2                                  # position of sequence 0: later tokens see it, earlier ones do not
    page, row = c.table_np[0, bad // P], bad % P
    for what in (float("nan"), float("inf"), -float("inf")):
        kept = c.v_pages[page, :, row].clone(), c.k_pages[page, :, row].clone()
        c.v_pages[page, :, row, 3:5] = what
        out, lse = c.attend(q)
        clean = torch.ones(c.T, dtype=torch.bool, device=DEV)
        clean[new // 2:new] = False
        assert not torch.isfinite(out[new // 2:new, :, 3:5].float()).any()
        c.v_pages[page, :, row] = kept[0]
        close(c, q, out, lse, rows=clean)
        c.k_pages[page, :, row] = what
        out, lse = c.attend(q)
        c.k_pages[page, :, row] = kept[1]
        close(c, q, out, lse, rows=clean)


@gpu
@pytest.mark.parametrize("dtype,D,P,new", [("bf16", 128, 16, 2), ("bf16", 128, 16, 40), ("bf16", 128, 24, 300), ("bf16", 40, 9, 3), ("f32", 64, 16, 2)])
def test_sequences_and_pages_that_are_not_valid(dtype, D, P, new):
    """Whatever the arrays hold, nothing is read or written outside the pools: the sequence is skipped, the page read as zeros."""
    lens = [(100, new), (60, new), (33, new), (200, new)]
    c = Cache(dtype, 4, 2, D, P, lens, seed=3, extra_rows=5, rot=D)
    rows = c.rand(c.T, 8, D)
    q = rows[:, :4]
    good, lse = c.attend(q)
    c.check(q, good, lse)
    # a page entry outside the pool
    c.table_np[1, 1] = c.k_pages.shape[0] + 3
    c.table_np[2, 0] = -1
    c.table.copy_(torch.from_numpy(c.table_np))
    out, lse = c.attend(q)
    c.check(q, out, lse)
    assert int(c.status.item()) == c.b.MRP_DEV_BAD_INDEX
    assert c.b.mrp_fetch_status(c.ctx, clear=True) == c.b.MRP_DEV_BAD_INDEX
    c.status.zero_()
    k0, v0 = f64(c.k_pages), f64(c.v_pages)
    qo = torch.full((c.T, 4, D), 7.0, device=DEV, dtype=TORCH[dtype])
    c.b.mrp_kv_append(c.ctx, c.batch, c.k_pages, c.v_pages, rows[:, 4:6], rows[:, 6:8], None, q, qo)
    kp, vp = ref.append(k0, v0, np.zeros((c.T, 2, D)), f64(rows[:, 6:8]), c.start_np, c.pre_np, c.table_np, P)
    assert np.array_equal(f64(c.v_pages), vp, equal_nan=True)
    # lengths that do not fit: a negative one, one beyond the table, rows beyond the arrays, a start behind its end
    for pre, start in (([-1, 60, 33, 200], None), ([100, 10 ** 9, 33, 200], None), ([2 ** 31 - 1, 60, 33, 200], None),
                       (None, [0, new, 2 * new, 3 * new, c.T + 9]), (None, [0, new, new - 1, 3 * new, 4 * new]), (None, [-4, new, 2 * new, 3 * new, 4 * new])):
        c.status.zero_()
        p0, s0 = c.pre_np, c.start_np
        c.pre_np = np.array(pre, np.int32) if pre else p0
        c.start_np = np.array(start, np.int32) if start else s0
        c.prefix_len.copy_(torch.from_numpy(c.pre_np))
        c.seq_start.copy_(torch.from_numpy(c.start_np))
        out, lse = c.attend(q)
        if not (start and start[2] < start[1]):            # (there two sequences claim the same rows)
            c.check(q, out, lse)
        assert int(c.status.item()) & c.b.MRP_DEV_BAD_INDEX
        before = c.v_pages.clone()
        c.status.zero_()
        c.b.mrp_kv_append(c.ctx, c.batch, c.k_pages, c.v_pages, rows[:, 4:6], rows[:, 6:8] + 1, None, q, qo)
        _, vp = ref.append(f64(before), f64(before), np.zeros((c.T, 2, D)), f64(rows[:, 6:8] + 1), c.start_np, c.pre_np, c.table_np, P)
        if not (start and start[2] < start[1]):
            assert np.array_equal(f64(c.v_pages), vp, equal_nan=True)
        assert int(c.status.item()) & c.b.MRP_DEV_BAD_INDEX
        c.pre_np, c.start_np = p0, s0
        c.prefix_len.copy_(torch.from_numpy(p0))
        c.seq_start.copy_(torch.from_numpy(s0))
    c.b.mrp_fetch_status(c.ctx, clear=True)
    c.status.zero_()
    c.attend(q)
    assert int(c.status.item()) == c.b.MRP_DEV_BAD_INDEX    # (the two page entries of above)


@gpu
@pytest.mark.parametrize("start", [[0, 99, 4, 8, 12], [0, 99, 1, 2, 5], [0, 8, 4, 8, 12], [99, 0, 4, 7, 7], [0, 4, 99, -1, 6], [0, 2, 100, 1, 9]])
@pytest.mark.parametrize("new", [1, 5])
def test_lists_of_rows_that_do_not_ascend(start, new):
    """Sequences that do not fit make the list of starts rise and fall: the others keep their rows, no row goes elsewhere."""
    c = Cache("bf16", 4, 2, 64, 16, [(15, 4), (40, 4), (31, 4), (30, 4)], seed=9, extra_rows=3, rot=64)
    c.batch.c.max_new = new
    rows = c.rand(c.T, 8, 64)
    c.start_np = np.array(start, np.int32)
    c.seq_start.copy_(torch.from_numpy(c.start_np))
    taken = [s + i for _, s, n, _ in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * 16) for i in range(n)]
    before = f64(c.v_pages)
    qo = torch.full((c.T, 4, 64), 7.0, device=DEV, dtype=torch.bfloat16)
    c.b.mrp_kv_append(c.ctx, c.batch, c.k_pages, c.v_pages, rows[:, 4:6], rows[:, 6:8], None, rows[:, :4], qo)
    _, vp = ref.append(before, before, np.zeros((c.T, 2, 64)), f64(rows[:, 6:8]), c.start_np, c.pre_np, c.table_np, 16)
    if len(set(taken)) == len(taken):                      # (else two sequences claim a row)
        assert np.array_equal(f64(c.v_pages), vp, equal_nan=True)
        out, lse = c.attend(qo)
        c.check(qo, out, lse)
    wrote = (f64(qo) != 7.0).any((1, 2))
    assert np.array_equal(np.flatnonzero(wrote), np.unique(taken))
    assert int(c.status.item()) == c.b.MRP_DEV_BAD_INDEX


@gpu
@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 20), ("bf16", 150), ("f32", 3)])
def test_attention_in_place(dtype, new):
    c = Cache(dtype, 8, 2, 128, 16, [(3000, new), (70, new), (0, new)], seed=5)
    q = c.rand(c.T, 8, 128)
    out, lse = c.attend(q)
    c.check(q, out, lse)
    same = q.clone()
    again, lse2 = c.attend(same, same)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


@gpu
@pytest.mark.parametrize("gap", [8, 1024, 4096 + 1024])
@pytest.mark.parametrize("D,P,new", [(128, 16, 1), (128, 24, 9), (128, 32, 40), (256, 8, 2), (256, 96, 40), (128, 16, 200)])
def test_small_pages_with_gaps(D, P, new, gap):
    c = Cache("bf16", 4, 2, D, P, [(500, new), (P - 1, new), (1, new)], seed=7, page_gap=gap)
    q = c.rand(c.T, 4, D)
    out, lse = c.attend(q)
    c.check(q, out, lse)


@gpu
@pytest.mark.parametrize("dtype,D,new", [("bf16", 128, 1), ("bf16", 128, 24), ("bf16", 64, 150), ("f32", 64, 3)])
def test_a_captured_step_serves_other_lengths(dtype, D, new):
    c = Cache(dtype, 4, 2, D, 16, [(700, new), (64, new), (300, new)], seed=8, rot=D)
    rows = c.rand(c.T, 8, D)
    q, out, lse = torch.empty((c.T, 4, D), device=DEV, dtype=TORCH[dtype]), torch.empty((c.T, 4, D), device=DEV, dtype=TORCH[dtype]), torch.empty((c.T, 4), device=DEV)

    def step():
        c.b.mrp_kv_append(c.ctx, c.batch, c.k_pages, c.v_pages, rows[:, 4:6], rows[:, 6:8], None, rows[:, :4], q)
        c.attend(q, out, lse=False)
        c.b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, q, out, lse)
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
        for b, p in enumerate(pre):                       # the cached positions hold values, what lies behind them is junk again
            for j0 in range(0, c.lens[b][0] + new, 16):
                for pool in (c.k_pages, c.v_pages):
                    page = c.rand(2, 16, D)
                    page[:, max(0, p - j0):] = float("nan")
                    pool[c.table_np[b, j0 // 16]] = page
        graph.replay()
        torch.cuda.synchronize()
        c.lens = [(p, new) for p in pre]
        c.check(q, out, lse)
        want, wl = out.clone(), lse.clone()
        step()                                            # the same call, not captured
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl)
        c.lens = [(700, new), (64, new), (300, new)]
    assert int(c.status.item()) == 0


@gpu
def test_two_contexts_on_two_streams_at_once():
    cs = [Cache("bf16", 32, 8, 128, 16, [(1500, n), (900, n), (30, n)], seed=n) for n in (1, 40)]
    qs = [c.rand(c.T, 32, 128) for c in cs]
    want = [c.attend(q) for c, q in zip(cs, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    got = [[] for _ in cs]
    for _ in range(20):
        for i, (c, q, s) in enumerate(zip(cs, qs, streams)):
            out, lse = torch.full_like(want[i][0], 7.0), torch.full_like(want[i][1], 7.0)
            s.wait_stream(torch.cuda.current_stream())
            c.b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, q, out, lse, stream=s)
            got[i].append((out, lse))
    torch.cuda.synchronize()
    for i in range(2):
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
    cs[0].check(qs[0], *got[0][-1])


@gpu
@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("P", [16, 20])
def test_offsets_beyond_32_bits(new, P):
    """Pages 2^31 elements apart: a pool of which little is touched."""
    lens = [(3 * P - 1, new)]
    c = Cache("bf16", 4, 2, 128, P, lens, seed=4, spare_pages=0, rot=128)
    n_pages, page = c.k_pages.shape[0], 2 * P * 128
    stride = 2 ** 31 // max(1, n_pages - 2)
    stride -= stride % 8
    c.b.mrp_kv_attach(c.ctx, 4, 2, 128, P, n_pages, c.max_pages, stride, 128)
    pools = []
    for pool in (c.k_pages, c.v_pages):
        big = torch.empty((n_pages - 1) * stride + page, device=DEV, dtype=torch.bfloat16).as_strided((n_pages, 2, P, 128), (stride, P * 128, 128, 1))
        big.copy_(pool)
        pools.append(big)
    assert (n_pages - 1) * stride > 2 ** 31
    c.k_pages, c.v_pages = pools
    rows = c.rand(c.T, 8, 128)
    q = torch.empty((c.T, 4, 128), device=DEV, dtype=torch.bfloat16)
    c.b.mrp_kv_append(c.ctx, c.batch, c.k_pages, c.v_pages, rows[:, 4:6], rows[:, 6:8], None, rows[:, :4], q)
    out, lse = c.attend(q)
    c.check(q, out, lse)
    assert torch.equal(c.v_pages[c.table_np[0, (3 * P - 1) // P], :, (3 * P - 1) % P], rows[0, 6:8])


@gpu
@pytest.mark.parametrize("new", [2, 30, 140])
def test_strided_rows_and_rows_of_no_sequence(new):
    c = Cache("bf16", 6, 2, 64, 16, [(50, new), (3, new)], seed=6, extra_rows=4)
    wide = c.rand(c.T, 6 + 4, 64)
    q = wide[:, 2:8]
    store = torch.full((c.T, 9, 64), 7.0, device=DEV, dtype=torch.bfloat16)
    out, lse = c.attend(q, store[:, 1:7])
    c.check(q, out, lse)
    assert (store[:, 0] == 7).all() and (store[:, 7:] == 7).all() and (store[-4:] == 7).all()
    dense_out, dense_lse = c.attend(q.contiguous())
    assert torch.equal(dense_out, out) and torch.equal(dense_lse, lse)
    assert torch.equal(c.attend(q, lse=False)[0], out)


@gpu
def test_empty_batches_and_empty_sequences():
    c = Cache("bf16", 4, 2, 128, 16, [(20, 0), (30, 3), (0, 0)], seed=1)
    q = c.rand(c.T, 4, 128)
    out, lse = c.attend(q)
    c.check(q, out, lse)
    none = c.b.KvBatch(c.seq_start[:1], c.prefix_len[:0], c.table[:0], 0, 0)
    out = torch.full((3, 4, 128), 7.0, device=DEV, dtype=torch.bfloat16)
    c.b.mrp_paged_attention(c.ctx, none, c.k_pages, c.v_pages, q, out)
    c.b.mrp_kv_append(c.ctx, none, c.k_pages, c.v_pages, q[:, :2], q[:, :2])
    assert c.ctx.last_launch_count == 0
    c.b.mrp_qk_norm_rotate(c.ctx, None, q[:0], None, out[:0], None)
    torch.cuda.synchronize()
    assert (out == 7).all()
    zeros = torch.zeros(2, dtype=torch.int32, device=DEV)          # sequences, but not a token among them
    b = c.b.KvBatch(zeros, zeros[:1], c.table[:1], 3, 1)
    c.b.mrp_paged_attention(c.ctx, b, c.k_pages, c.v_pages, q, out)
    torch.cuda.synchronize()
    assert (out == 7).all()


@gpu
def test_the_tile_kernels_agree_with_the_few_row_kernel():
    lens = [(333, 40), (900, 2), (0, 129)]
    c = Cache("bf16", 8, 2, 128, 32, lens, seed=12)
    q = c.rand(c.T, 8, 128)
    out, lse = c.attend(q)
    w_lm = torch.zeros((32, 64), device=DEV, dtype=torch.bfloat16)
    other = c.b.mrp_create(64, 64, 32, [], w_lm, max_rows=1, max_seqs=3, block_len=1, flags=c.b.MRP_FLAG_FORCE_SIMT)
    c.b.mrp_kv_attach(other, 8, 2, 128, 32, c.k_pages.shape[0], c.max_pages)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    c.b.mrp_paged_attention(other, c.batch, c.k_pages, c.v_pages, q, o2, l2)
    close(c, q, o2, l2)
    close(c, q, out, lse)
    assert (lse - l2).abs().max() < 1e-4


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_decoding_loop(dtype):
    """Prompts and blocks: norm and rotation on the way into the cache, every block decoded twice (its rows overwritten) and
    then committed; against one 64-bit pass over each whole sequence."""
    H, Hk, D, P, B, L = 8, 2, 64, 16, 3, 4
    first = [70, 1, 33]
    steps = 3
    total = [n + steps * L for n in first]
    c = Cache(dtype, H, Hk, D, P, [(0, t) for t in total], seed=2, rot=D, theta=1e4)
    for pool in (c.k_pages, c.v_pages):
        pool.fill_(float("nan"))
    gq, gk = 1 + 0.2 * c.rand(D), 1 + 0.2 * c.rand(D)
    feed = [c.rand(t, H + 2 * Hk, D) for t in total]       # what the projection gives for each position
    done, results = [0] * B, [[] for _ in range(B)]
    start = [0] * B
    for it in range(steps + 1):
        new = first if it == 0 else [L] * B
        seq_start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
        pre = torch.tensor(done, dtype=torch.int32, device=DEV)
        batch = c.b.KvBatch(seq_start, pre, c.table, sum(new), max(new))
        for attempt in range(2 if it else 1):
            rows = torch.cat([feed[b][done[b]:done[b] + new[b]] for b in range(B)])
            if attempt == 0 and it:
                rows = c.rand(*rows.shape)                # a first guess at the block: overwritten by the second
            q, out, lse = (torch.empty((sum(new), H, D), device=DEV, dtype=TORCH[dtype]) for _ in range(2)), None, None
            qn, out = q
            lse = torch.empty((sum(new), H), device=DEV)
            c.b.mrp_kv_append(c.ctx, batch, c.k_pages, c.v_pages, rows[:, H:H + Hk], rows[:, H + Hk:], gk, rows[:, :H], qn, gq)
            c.b.mrp_paged_attention(c.ctx, batch, c.k_pages, c.v_pages, qn, out, lse)
        for b in range(B):
            results[b].append((out[seq_start[b]:seq_start[b + 1]], lse[seq_start[b]:seq_start[b + 1]], qn[seq_start[b]:seq_start[b + 1]]))
            done[b] += new[b]
    torch.cuda.synchronize()
    out, lse, qn = (torch.cat([torch.cat([r[i] for r in results[b]]) for b in range(B)]) for i in range(3))
    close(c, qn, out, lse)                                # attention over what the cache now holds
    for b in range(B):                                    # and what it holds is the rotated feed
        pages = torch.from_numpy(c.table_np[b, :-(-total[b] // P)].astype(np.int64)).to(DEV)
        got = c.k_pages[pages].permute(0, 2, 1, 3).reshape(-1, Hk, D)[:total[b]]
        want = ref.norm_rotate(f64(feed[b][:, H:H + Hk]), np.arange(total[b]), f64(gk), D, 1e4)
        assert (np.abs(f64(got) - want) <= 4 * (D / 2 + 16) * U * np.abs(want).max() + half_step(dtype) * np.abs(want)).all()
        assert torch.equal(c.v_pages[pages].permute(0, 2, 1, 3).reshape(-1, Hk, D)[:total[b]], feed[b][:, H + Hk:])


@gpu
def test_prefix_and_block_join_by_their_log_sums():
    c = Cache("f32", 4, 2, 64, 16, [(100, 8), (37, 8), (0, 8)], seed=21)
    q = c.rand(c.T, 4, 64)
    whole, lw = c.attend(q, mask=c.b.MRP_ATTN_BLOCK)
    a, la = c.attend(q, mask=c.b.MRP_ATTN_PREFIX)
    # the block's own keys: a cache that begins at the block
    o, l = torch.zeros_like(whole).double(), torch.zeros_like(lw).double()
    for b in range(3):
        p, s = c.lens[b][0], int(c.start_np[b])
        k, v = (torch.stack([pool[c.table_np[b, (p + j) // 16], :, (p + j) % 16] for j in range(8)], 1).double().repeat_interleave(2, 0) for pool in (c.k_pages, c.v_pages))
        z = torch.einsum("nhd,hjd->nhj", q[s:s + 8].double(), k) / 8.0
        l[s:s + 8] = torch.logsumexp(z, -1)
        o[s:s + 8] = torch.einsum("nhj,hjd->nhd", torch.softmax(z, -1), v)
    m = torch.logaddexp(la.double(), l)
    joined = a.double() * (la.double() - m).exp()[..., None] + o * (l - m).exp()[..., None]
    assert (m - lw.double()).abs().max() < 1e-5
    assert (joined - whole.double()).abs().max() < 1e-5


@gpu
def test_prefix_caches_of_the_module_are_such_a_pool():
    """mrp_module_set_prefix's caches [max_seqs, heads, cap, d / heads] = a pool of max_seqs pages of cap rows."""
    from paper_2605_18817_b200 import binding
    B, heads, dh, cap = 3, 4, 64, 200
    d = heads * dh
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    r = lambda *s: (torch.randn(s, generator=g, device=DEV) * 0.05).to(torch.bfloat16)        # noqa: E731
    ctx = binding.mrp_create(d, 256, 512, [], r(512, d), max_rows=B * 4, max_seqs=B, block_len=4)
    layer = dict(g_attn=1 + r(d), w_q=r(d, d), w_k=r(d, d), w_v=r(d, d), w_o=r(d, d), g_mlp=1 + r(d), w_gate=r(256, d), w_up=r(256, d), w_down=r(d, 256))
    binding.mrp_module_attach(ctx, r(512, d), r(d, 2 * d), [layer], heads, 0)
    k, v = (torch.zeros((B, heads, cap, dh), device=DEV, dtype=torch.bfloat16) for _ in range(2))
    plen = torch.zeros(B, dtype=torch.int32, device=DEV)
    binding.mrp_module_set_prefix(ctx, [(k, v)], plen, append=True)
    tokens, conf, lse, tok = torch.zeros(B * 4, dtype=torch.int32, device=DEV), *(torch.empty((2, 12), device=DEV) for _ in range(2)), torch.empty((2, 12), dtype=torch.int32, device=DEV)
    for step in range(9):                                 # nine blocks committed to the module's prefix
        binding.mrp_module_step(ctx, tokens + step, r(B * 4, d) * 20, torch.empty((B * 4, d), device=DEV), torch.zeros((B * 4, 512), device=DEV), None,
                                12, B, 4, True, conf, lse, tok)
        plen += 4
    torch.cuda.synchronize()
    assert (k[:, :, :36].float().abs().sum((1, 3)) > 0).all() and (k[:, :, 36:] == 0).all()
    binding.mrp_kv_attach(ctx, heads, heads, dh, cap, n_pages=B, max_pages=1)
    table = torch.arange(B, dtype=torch.int32, device=DEV)[:, None].contiguous()
    start = torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device=DEV)
    q, out, l = r(2 * B, heads, dh) * 20, torch.empty((2 * B, heads, dh), device=DEV, dtype=torch.bfloat16), torch.empty((2 * B, heads), device=DEV)
    binding.mrp_paged_attention(ctx, binding.KvBatch(start, plen, table, 2 * B, 2), k, v, q, out, l, mask=binding.MRP_ATTN_PREFIX)
    want, wl, reach, size = ref.attention(f64(q), f64(k), f64(v), start.cpu().numpy(), plen.cpu().numpy(), table.cpu().numpy(), cap, ref.PREFIX)
    z = (dh * U) * size + 4 * U * (size + 1)
    assert (np.abs(f64(out) - want) <= reach * (2 * z + 72 * U + 2.0 ** -8)[..., None] + 2.0 ** -8 * np.abs(want)).all()
    assert (np.abs(f64(l) - wl) <= z + 36 * U + 4 * U * (np.abs(wl) + 1)).all()
    binding.mrp_destroy(ctx)


@gpu
def test_refusals():
    c = Cache("bf16", 4, 2, 128, 16, [(20, 3)], seed=1, rot=128)
    b, q = c.b, c.rand(3, 4, 128)
    out = torch.empty_like(q)

    def status(fn):
        with pytest.raises(b.MrpError) as e:
            fn()
        return e.value.status
    att = lambda **kw: b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, q, out, **kw)         # noqa: E731
    for kw in (dict(mask=3), dict(mask=-1), dict(window=-1), dict(sinks=-2), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-1.0)):
        assert status(lambda: att(**kw)) == 1
    fresh = b.mrp_create(64, 64, 32, [], torch.zeros((32, 64), device=DEV, dtype=torch.bfloat16), max_rows=1, max_seqs=1, block_len=1)
    assert status(lambda: b.mrp_paged_attention(fresh, c.batch, c.k_pages, c.v_pages, q, out)) == 2
    b.mrp_kv_attach(fresh, 4, 2, 128, 16)                  # no cache: the rotation alone
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)
    b.mrp_qk_norm_rotate(fresh, pos, q, None, out, None)
    assert torch.equal(out, q)
    with pytest.raises(ValueError):
        b.mrp_paged_attention(fresh, c.batch, c.k_pages, c.v_pages, q, out)
    assert status(lambda: b.mrp_qk_norm_rotate(c.ctx, None, q, None, out, None)) == 1        # a rotation without positions
    two = b.KvBatch(torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), c.table.repeat(2, 1), 0, 0)
    assert status(lambda: b.mrp_paged_attention(c.ctx, two, c.k_pages, c.v_pages, q, out)) == 1         # more than max_seqs
    for bad in (q.float(), q[:, :3], q[:2], q.transpose(0, 1), q.cpu()):
        with pytest.raises((TypeError, ValueError)):
            b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, bad, out)
    for bad in (c.k_pages[:-1], c.k_pages.float(), c.k_pages.transpose(1, 2)):
        with pytest.raises((TypeError, ValueError)):
            b.mrp_paged_attention(c.ctx, c.batch, bad, c.v_pages, q, out)
    with pytest.raises(TypeError):
        b.KvBatch(c.seq_start.long(), c.prefix_len, c.table, 3, 3)
    with pytest.raises(ValueError):
        b.KvBatch(c.seq_start[:1], c.prefix_len, c.table, 3, 3)
    # unaligned rows, rows that overlap, in place with other strides
    store = torch.zeros(3 * 4 * 128 + 64, device=DEV, dtype=torch.bfloat16)
    assert status(lambda: b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, store[4:4 + 1536].view(3, 4, 128), out)) == 1
    assert status(lambda: b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, store.as_strided((3, 4, 128), (504, 128, 1)), out)) == 1
    assert status(lambda: b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, store.as_strided((3, 4, 128), (516, 128, 1)), out)) == 1
    wide = torch.zeros((3, 5, 128), device=DEV, dtype=torch.bfloat16)
    r = b.mrp_qkv_rows(wide.data_ptr(), None, None, 640, 0, 0, None, None, wide.data_ptr(), None, 512, 0)
    assert b.lib.mrp_qk_norm_rotate(c.ctx.handle, pos.data_ptr(), 3, ctypes.byref(r), None) == 1
    a = b.mrp_attention_args(wide.data_ptr(), wide.data_ptr(), 640, 512, None, 0, 0, 0, 0.0)
    pools = b.mrp_module_kv(c.k_pages.data_ptr(), c.v_pages.data_ptr())
    assert b.lib.mrp_paged_attention(c.ctx.handle, c.batch.ref, ctypes.byref(pools), ctypes.byref(a), None) == 1
    for kw in (dict(n_heads=3), dict(head_dim=12), dict(head_dim=264), dict(page_size=0), dict(n_pages=-1), dict(max_pages=0), dict(page_stride=100),
               dict(page_stride=4100), dict(rot_dim=3), dict(rot_dim=130), dict(rot_theta=0.0), dict(norm_eps=-1.0), dict(inv_freq=[float("inf")] * 64)):
        a = dict(n_heads=4, n_kv_heads=2, head_dim=128, page_size=16, n_pages=4, max_pages=4, rot_dim=128, rot_theta=1e4)
        a.update(kw)
        assert status(lambda: b.mrp_kv_attach(fresh, **a)) == 1
    cfg = b.mrp_kv_config(4, 2, 128, 16, 4, 4, 0, 0, 0, 1e4, None, 1e-6)
    ws = torch.empty(256, dtype=torch.uint8, device=DEV)
    assert b.lib.mrp_kv_attach(fresh.handle, ctypes.byref(cfg), ctypes.c_void_p((ws.data_ptr() + 255) // 256 * 256), 0) == 4
    assert b.lib.mrp_kv_attach(fresh.handle, ctypes.byref(cfg), ctypes.c_void_p(ws.data_ptr() // 256 * 256 + 8), 1 << 30) == 1
    out2, lse2 = c.attend(q)                              # nothing of this has touched the context
    c.check(q, out2, lse2)


def test_refusals_on_the_host():
    from paper_2605_18817_b200 import binding as b
    lib = b.lib
    assert lib.mrp_kv_attach(None, None, None, 0) == 1
    assert lib.mrp_qk_norm_rotate(None, None, 1, None, None) == 1
    assert lib.mrp_kv_append(None, None, None, None, None) == 1
    assert lib.mrp_paged_attention(None, None, None, None, None) == 1
    cfg = b.mrp_config(64, 64, 32, 0, 1, 4, 1, b.MRP_BF16, 1e-6, 0, 0)
    good = dict(n_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10, max_pages=4, page_stride=0, rot_dim=64, rot_interleaved=0,
                rot_theta=1e4, inv_freq=None, norm_eps=1e-6)

    def size(**kw):
        a = dict(good)
        a.update(kw)
        return int(lib.mrp_kv_workspace_bytes(ctypes.byref(cfg), ctypes.byref(b.mrp_kv_config(*a.values()))))
    assert size() > 0 and size(n_pages=0, max_pages=0) > 0 and size(page_stride=2 * 16 * 128 + 8) > 0 and size(head_dim=256) > 0
    for kw in (dict(n_heads=0), dict(n_kv_heads=3), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=100), dict(head_dim=264), dict(page_size=0),
               dict(n_pages=-1), dict(max_pages=0), dict(max_pages=1 << 27), dict(page_stride=8), dict(page_stride=2 * 16 * 128 + 4), dict(rot_dim=-2),
               dict(rot_dim=65), dict(rot_dim=130), dict(rot_theta=0.0), dict(rot_theta=float("inf")), dict(norm_eps=-1.0), dict(norm_eps=float("nan")),
               dict(page_stride=1 << 59)):
        assert size(**kw) == 0, kw
    assert int(lib.mrp_kv_workspace_bytes(None, None)) == 0

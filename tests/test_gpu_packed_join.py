"""Joining where nothing may change: a pass that saw nothing leaves the own keys' rows as they are, bit for bit, and one that outweighs them
by more than fp32 holds stays as it was, bit for bit.  And one window over a cache and the block behind it, by two passes."""
import math

import numpy as np
import pytest
import torch

from test_gpu_kv import DEV, U, Cache, half_step
from test_gpu_q8 import CacheQ8, Rows

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("H,Hk,D,new,mask,window,sinks", [
    (8, 2, 128, [4, 4, 1, 0, 33], 1, 0, 0), (8, 2, 128, [300, 1, 130], 0, 0, 0), (5, 1, 80, [33, 2, 70], 0, 9, 2), (4, 2, 256, [130, 3], 1, 0, 0),
    (3, 3, 8, [20, 65], 0, 0, 0), (32, 8, 64, [90] * 30, 0, 0, 0)], ids=str)
@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", "16-row tiles"), ("f32", 0)])
def test_rows_that_a_join_leaves_as_they_are(dtype, flags, H, Hk, D, new, mask, window, sinks):
    from paper_2605_18817_b200 import binding
    c = Rows(dtype, H, Hk, D, new, seed=4, extra_rows=2, flags=binding.MRP_FLAG_FORCE_SIMT if flags else 0)
    mine = torch.zeros(c.T, dtype=torch.bool, device=DEV)
    mine[:int(c.start_np[-1])] = True
    kw = dict(mask=mask, window=window, sinks=sinks)
    for hint in (max(new), 1, 10000):
        c.batch.c.max_new = hint
        alone, la = c.attend(**kw)
        c.close(alone, la, **kw)
        # nothing seen by the other pass: whatever its rows hold is not read
        for junk in (float("nan"), float("inf"), 3.0):
            out, lse = torch.full_like(alone, junk), torch.full_like(la, -math.inf)
            c.attend(out, lse, join=True, **kw)
            assert torch.equal(out[mine], alone[mine]) and torch.equal(lse[mine], la[mine])
            assert torch.isneginf(lse[~mine]).all() and torch.equal(out[~mine].nan_to_num(5.0), torch.full_like(out[~mine], junk).nan_to_num(5.0))
        # 2^-150 of the other pass's weight is nothing: e^(-400) < 2^-577
        prior, pl = c.rand(c.T, H, D), la + 400.0
        out, lse = prior.clone(), pl.clone()
        c.attend(out, lse, join=True, **kw)
        assert torch.equal(out, prior)
        # (to base 2 and back: a rounding of the factor, of the product and of each way back)
        assert ((lse - pl).abs() <= 4 * U * pl.abs()).all()
    assert int(c.status.item()) == 0


@gpu
@pytest.mark.parametrize("kind", ["as it is", "8 bits"])
@pytest.mark.parametrize("dtype,H,Hk,D,P,lens,window,sinks", [
    ("bf16", 8, 2, 128, 16, [(300, 32), (40, 9), (7, 32)], 20, 5), ("bf16", 8, 2, 128, 16, [(300, 4), (17, 3)], 2, 1), ("bf16", 4, 1, 80, 9, [(100, 40)], 33, 64),
    ("f32", 4, 2, 64, 16, [(90, 12), (3, 20)], 6, 3), ("bf16", 32, 8, 64, 32, [(500, 200), (200, 130)], 150, 4)], ids=str)
def test_one_window_over_cache_and_block(kind, dtype, H, Hk, D, P, lens, window, sinks):
    """A window shorter or longer than the block, with first tokens: the join's own pass takes sinks 0."""
    c = (Cache if kind == "as it is" else CacheQ8)(dtype, H, Hk, D, P, lens, seed=8)
    rows = c.rand(c.T, H + 2 * Hk, D)
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    r, split = half_step(dtype), 0.0 if dtype == "bf16" else 2.0 ** -20
    for mask in (c.b.MRP_ATTN_BLOCK, c.b.MRP_ATTN_CAUSAL):
        out, lse = c.attend(q, mask=c.b.MRP_ATTN_PREFIX, window=window, sinks=sinks)
        c.b.mrp_packed_attention(c.ctx, c.batch, k, v, q, out, lse, mask=mask, window=window, sinks=0, join=True)
        for b, ((p, n), s) in enumerate(zip(lens, c.start_np)):
            assert p >= sinks
            pages = torch.from_numpy(c.table_np[b, :-(-p // P)].astype(np.int64)).to(DEV)
            held = [pool[pages].double().permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :p] for pool in (c.k_pages, c.v_pages)]
            kk, vv = (torch.cat([h, x[s:s + n].double().transpose(0, 1)], 1).repeat_interleave(H // Hk, 0) for h, x in zip(held, (k, v)))
            x, pos, j = q[s:s + n].double().transpose(0, 1), p + torch.arange(n, device=DEV)[:, None], torch.arange(p + n, device=DEV)
            seen = ((j <= pos) if mask == c.b.MRP_ATTN_CAUSAL else (j >= 0)) & ((j > pos - window) | (j < sinks))
            zz = (x @ kk.transpose(1, 2) / math.sqrt(D)).masked_fill(~seen, -math.inf)
            w = torch.softmax(zz, -1)
            want, reach, lw = (w @ vv).transpose(0, 1), (w @ vv.abs()).transpose(0, 1), torch.logsumexp(zz, -1).T
            size = (x.abs() @ kk.abs().transpose(1, 2) / math.sqrt(D)).amax(-1).T
            z = (D * U + split) * size + 16 * U * (size + 2) + (p + n) * U
            # one rounding of the cache's part, one of the probabilities, one of the result
            tol = reach * (4 * z + (2 * r if dtype == "bf16" else 2 * split + r))[..., None] + r * want.abs()
            assert ((out[s:s + n].double() - want).abs() <= tol).all()
            assert ((lse[s:s + n].double() - lw).abs() <= 2 * z).all()
    assert int(c.status.item()) == 0

"""Joining where nothing may change: a pass that saw nothing leaves the own keys' rows as they are, bit for bit, and one that outweighs them
by more than fp32 holds stays as it was, bit for bit."""
import math

import pytest
import torch

from test_gpu_kv import DEV, U
from test_gpu_q8 import Rows

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

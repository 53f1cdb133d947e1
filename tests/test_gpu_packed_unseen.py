"""Packed attention: a value that is not finite reaches only the rows that see it, wherever the borders of a kernel's tiles of query rows
and keys fall: before a window, behind the diagonal, between the first tokens and the window.

A value: rows that do not see it give the bits that they give without it, since its probability is 0 and its row counts as zeros, and
adding 0 changes no sum; rows that see it are not finite where it is not.  A key: rows that do not see it are as close to the definition
as ever (the rows of a warp raise their maxima together, so they may round in other places); rows that see it are NaN."""
import pytest
import torch

from test_gpu_kv import DEV
from test_gpu_q8 import Rows

gpu = pytest.mark.gpu

# dtype, H, Hk, D, lengths, mask, window, sinks: rows of a sequence that go past a multiple of 16, 64 or 128 by less than a token's heads
UNSEEN = [
    ("bf16", 8, 1, 128, [9, 3], 0, 4, 0),
    ("bf16", 8, 1, 128, [9, 17], 1, 4, 0),
    ("bf16", 4, 1, 64, [17, 33, 49], 0, 1, 0),
    ("bf16", 8, 2, 128, [17, 33], 0, 9, 2),
    ("bf16", 2, 2, 128, [65, 1], 0, 4, 0),
    ("bf16", 1, 1, 256, [65, 129], 0, 4, 3),
    ("bf16", 2, 1, 80, [33, 70], 1, 5, 1),
    ("bf16", 64, 1, 64, [2, 3], 0, 0, 0),
    ("bf16", 64, 1, 128, [4], 1, 1, 0),
    ("bf16", 150, 1, 64, [1, 2, 3], 0, 0, 0),
    ("bf16", 150, 1, 64, [3], 0, 1, 1),
    ("bf16", 32, 8, 128, [33, 65, 130], 0, 20, 5),
    ("bf16", 4, 2, 128, [129, 257], 0, 100, 0),
    ("f32", 8, 1, 64, [9, 3], 0, 4, 0),
    ("f32", 4, 4, 40, [17, 65], 1, 4, 2),
    ("f32", 64, 1, 64, [2], 0, 0, 0),
]


def sees(i, j, n, mask, window, sinks):
    return (j <= i if mask == 0 else j < n) and (window == 0 or j > i - window or j < sinks)


@gpu
@pytest.mark.parametrize("flags", ["", "16-row tiles"])
@pytest.mark.parametrize("case", UNSEEN, ids=lambda c: "%s-H%d-%d-D%d-n%d-m%d-w%d-s%d" % (c[0], c[1], c[2], c[3], max(c[4]), c[5], c[6], c[7]))
def test_what_a_row_does_not_see_does_not_reach_it(case, flags):
    dtype, H, Hk, D, new, mask, window, sinks = case
    from paper_2605_18817_b200 import binding
    c = Rows(dtype, H, Hk, D, new, seed=D, extra_rows=1, flags=binding.MRP_FLAG_FORCE_SIMT if flags else 0)
    kw = dict(mask=mask, window=window, sinks=sinks)
    prior, pl = c.rand(c.T, H, D), c.rand(c.T, H).float()
    starts = [int(s) for s in c.start_np]
    mine = torch.arange(c.T, device=DEV) < starts[-1]
    for hint in (max(new), 1, 10000):                      # each kernel, whichever the lengths would choose
        c.batch.c.max_new = hint
        plain, lse = c.attend(**kw)
        c.close(plain, lse, **kw)
        joined, jl = prior.clone(), pl.clone()
        c.attend(joined, jl, join=True, **kw)
        for b, n in enumerate(new):
            s = starts[b]
            for j in sorted({0, 1, n // 3, n // 2, max(0, n - 2), n - 1} & set(range(n))):
                hit = torch.zeros(c.T, dtype=torch.bool, device=DEV)
                hit[s:s + n] = torch.tensor([sees(i, j, n, mask, window, sinks) for i in range(n)], device=DEV)
                good = c.v[s + j].clone()
                for what in (float("nan"), float("inf")):
                    c.v[s + j] = what
                    out, l2 = c.attend(**kw)
                    out2, l3 = prior.clone(), pl.clone()
                    c.attend(out2, l3, join=True, **kw)
                    c.v[s + j] = good
                    assert torch.equal(out[~hit], plain[~hit]) and torch.equal(out2[~hit], joined[~hit]), (hint, b, j, what)
                    assert not torch.isfinite(out[hit].float()).any() and not torch.isfinite(out2[hit].float()).any()
                    assert torch.equal(l2, lse) and torch.equal(l3, jl)        # log-sum-exps know nothing of values
                good = c.k[s + j].clone()
                c.k[s + j] = float("nan")
                out, l2 = c.attend(**kw)
                c.k[s + j] = good
                c.close(out, l2, rows=~hit & mine, **kw)
                assert (out[~mine] == 7).all() and (l2[~mine] == 7).all(), (hint, b, j)
                assert torch.isnan(out[hit].float()).all() and torch.isnan(l2[hit]).all()
    assert int(c.status.item()) == 0

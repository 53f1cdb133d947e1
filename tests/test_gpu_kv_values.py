"""What values that are not finite may change: the output of the rows that see them, not their log-sum-exp (it depends on scores
alone), and nothing of the rows that do not."""
import pytest
import torch

from test_gpu_kv import U, Cache, DEV
from test_gpu_kv_paths import close, dense

gpu = pytest.mark.gpu


def check_lse(c, q, lse, **kw):
    _, l, _, size = dense(c, q, **kw)
    n = max(p + m for p, m in c.lens) + 1
    z = (c.D * U + (0.0 if c.dtype == "bf16" else 2.0 ** -20)) * size + 4 * U * (size + 1)
    assert torch.isfinite(lse).all()
    assert ((lse.double() - l).abs() <= z + n * U + 4 * U * (l.abs() + 1)).all()


VALUES = [
    # dtype, H, Hk, D, P, lens, position of the value in sequence 0
    ("bf16", 4, 2, 64, 16, [(150, 4), (40, 3)], 152),                    # up to 16 rows
    ("bf16", 4, 2, 128, 16, [(2500, 5), (40, 3)], 2502),                 # (units cut in pieces)
    ("bf16", 4, 2, 256, 16, [(150, 5), (40, 3)], 152),
    ("bf16", 32, 16, 128, 32, [(300, 4)] * 20, 302),                     # (whole units)
    ("bf16", 4, 2, 64, 16, [(150, 40), (40, 9)], 170),                   # one row tile
    ("bf16", 4, 2, 128, 64, [(2500, 40), (40, 9)], 2520),
    ("bf16", 4, 2, 256, 16, [(150, 40), (40, 9)], 170),
    ("bf16", 32, 16, 128, 32, [(300, 40)] * 12, 320),
    ("bf16", 64, 8, 64, 32, [(300, 20)] * 20, 310),                      # two row tiles
    ("bf16", 64, 8, 128, 32, [(300, 20)] * 20, 310),
    ("bf16", 64, 8, 128, 32, [(0, 700), (2000, 130)], 350),
    ("bf16", 4, 2, 128, 20, [(150, 9), (40, 2)], 155),                   # tiles of 16 rows
    ("f32", 4, 2, 64, 16, [(150, 9), (40, 2)], 155),
]


@gpu
@pytest.mark.parametrize("where", ["some rows", "all rows"])
@pytest.mark.parametrize("case", VALUES, ids=lambda c: "%s-H%d-%d-D%d-P%d-n%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5])))
def test_the_log_sum_exp_does_not_depend_on_values(case, where):
    dtype, H, Hk, D, P, lens, at = case
    c = Cache(dtype, H, Hk, D, P, lens, seed=D)
    q = c.rand(c.T, H, D)
    if where == "all rows":
        at = lens[0][0] // 2
    page, row = c.table_np[0, at // P], at % P
    kept = c.v_pages[page, :, row].clone()
    for what in (float("nan"), float("inf"), -float("inf")):
        c.v_pages[page, :, row, 3:5] = what
        out, lse = c.attend(q)
        clean = torch.ones(c.T, dtype=torch.bool, device=DEV)
        clean[max(0, at - lens[0][0]):lens[0][1]] = False
        assert not torch.isfinite(out[~clean][..., 3:5].float()).any()
        check_lse(c, q, lse)
        c.v_pages[page, :, row] = kept
        close(c, q, out, lse, rows=clean)


@gpu
@pytest.mark.parametrize("dtype,D,P,new", [("f32", 64, 16, 9), ("f32", 128, 24, 30), ("f32", 256, 16, 12), ("bf16", 64, 20, 9), ("bf16", 128, 16, 3),
                                           ("bf16", 128, 16, 40), ("bf16", 64, 32, 40)])
def test_the_types_extreme_values_reach_only_the_rows_that_see_them(dtype, D, P, new):
    """Finite, but at the end of the type's range: rows that do not see them are as they would be."""
    c = Cache(dtype, 4, 2, D, P, [(150, new), (40, new)], seed=D)
    q = c.rand(c.T, 4, D)
    page, row = c.table_np[0, (150 + new // 2) // P], (150 + new // 2) % P
    limits = torch.finfo(q.dtype)
    clean = torch.ones(c.T, dtype=torch.bool, device=DEV)
    clean[new // 2:new] = False
    kept = c.v_pages[page, :, row].clone(), c.k_pages[page, :, row].clone()
    for what in (limits.max, limits.min):
        c.v_pages[page, :, row] = what
        out, lse = c.attend(q)
        check_lse(c, q, lse)
        c.v_pages[page, :, row] = kept[0]
        close(c, q, out, lse, rows=clean)
        c.k_pages[page, :, row] = what
        out, lse = c.attend(q)
        c.k_pages[page, :, row] = kept[1]
        close(c, q, out, lse, rows=clean)

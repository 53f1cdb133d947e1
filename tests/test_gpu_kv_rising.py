"""Attention over the pages where scores rise along the cache: maxima grow from tile to tile, so sums and accumulators are
brought to new maxima again and again (inputs that are independent normals hardly ever do so behind a row's first tile).
Every kernel, whole and cut units, growth in all rows or in some; tolerances as in test_gpu_kv.py."""
import math

import pytest
import torch

from test_gpu_kv import Cache, DEV
from test_gpu_kv_paths import close

gpu = pytest.mark.gpu
LOG2E = 1.4426950408889634


def rising(c, rise, rows):
    """Queries for a cache whose scores rise by `rise` powers of two every 128 keys for the rows that look along feature 0.

    Keys: noise, and in feature 0 the height of their tile.  Queries: noise, and in feature 0 the row's part in the rise:
    "all" 1; "some" 1, 0, -1, 1/2 in turn (one that rises, one that does not, one that falls, one that rises half as fast)."""
    for b, (p, n) in enumerate(c.lens):
        for j in range(0, p + n, c.P):
            m = min(c.P, p + n - j)
            tile = torch.arange(j, j + m, device=DEV).div(128, rounding_mode="floor")
            c.k_pages[c.table_np[b, j // c.P], :, :m, 0] = (tile * (rise * math.sqrt(c.D) / LOG2E)).to(c.k_pages.dtype)
    q = c.rand(c.T, c.H, c.D)
    parts = torch.tensor([1.0] if rows == "all" else [1.0, 0.0, -1.0, 0.5], device=DEV)
    at = torch.arange(c.T, device=DEV)[:, None] + torch.arange(c.H, device=DEV)
    q[..., 0] = parts[at % len(parts)].to(q.dtype)
    return q


RISING = [
    # dtype, H, Hk, D, P, lens, mask
    ("bf16", 8, 2, 64, 16, [(2600, 2), (1500, 1)], 0),                  # up to 16 rows: transposed tiles, units cut in many pieces
    ("bf16", 8, 2, 128, 16, [(2600, 4), (1500, 3)], 0),
    ("bf16", 8, 2, 256, 32, [(2600, 4), (1500, 1)], 1),
    ("bf16", 16, 16, 128, 64, [(1900 - 100 * i, 1) for i in range(12)], 0),          # and whole ones
    ("bf16", 16, 4, 64, 16, [(2600, 20), (1500, 31)], 0),               # 17 to 128 rows: one row tile
    ("bf16", 16, 4, 128, 16, [(2600, 20), (1500, 31)], 0),
    ("bf16", 8, 2, 128, 64, [(2600, 10)], 1),                           # (one warp of rows has none)
    ("bf16", 16, 4, 256, 32, [(2600, 20), (1500, 31)], 0),
    ("bf16", 8, 1, 256, 64, [(900, 40), (0, 300)], 0),
    ("bf16", 64, 16, 128, 32, [(1400 - 100 * i, 24) for i in range(10)], 0),
    ("bf16", 64, 8, 64, 32, [(900 - 30 * i, 20) for i in range(20)], 0),             # more: two row tiles
    ("bf16", 64, 8, 128, 32, [(900 - 30 * i, 20) for i in range(20)], 0),
    ("bf16", 64, 8, 128, 64, [(0, 700), (2000, 130)], 0),
    ("bf16", 8, 2, 128, 20, [(1500, 2), (700, 9)], 0),                  # pages that boxes do not tile
    ("f32", 8, 2, 64, 16, [(1500, 3), (700, 9)], 0),
    ("f32", 4, 2, 128, 16, [(1500, 3), (700, 9)], 0),
    ("f32", 2, 2, 256, 16, [(1500, 2)], 0),
]


@gpu
@pytest.mark.parametrize("rise", [5, 9, 20])
@pytest.mark.parametrize("rows", ["all", "some"])
@pytest.mark.parametrize("case", RISING, ids=lambda c: "%s-H%d-%d-D%d-P%d-n%d" % (c[0], c[1], c[2], c[3], c[4], len(c[5])))
def test_maxima_that_grow_along_the_cache(case, rows, rise):
    dtype, H, Hk, D, P, lens, mask = case
    c = Cache(dtype, H, Hk, D, P, lens, seed=D + rise)
    q = rising(c, rise, rows)
    out, lse = c.attend(q, mask=mask)
    close(c, q, out, lse, mask=mask)
    for _ in range(20):
        again, lse2 = c.attend(q, mask=mask)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert int(c.status.item()) == 0

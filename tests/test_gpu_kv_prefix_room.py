"""The prefix mask attends to the cache alone, so a block whose own keys lie elsewhere needs no room behind its prefix: over a cache in the
context type as over one in 8 bits, and as the first pass of a join.  Tolerances as in test_gpu_kv.py; a joined row carries the
other pass's rounding beside its own."""
import math

import numpy as np
import pytest
import torch

from test_gpu_kv import DEV, TORCH, U, Cache, half_step
from test_gpu_kv_paths import close
from test_gpu_q8 import CacheQ8

gpu = pytest.mark.gpu

ROOM = [("f32", 4, 2, 64, 16, [(30, 40), (5, 90)]), ("f32", 3, 1, 8, 1, [(2, 9)]), ("bf16", 3, 1, 80, 7, [(20, 33), (0, 40)]),
        ("bf16", 2, 2, 128, 8, [(64, 16), (32, 12)]), ("bf16", 4, 2, 128, 16, [(60, 32), (64, 64)]), ("bf16", 2, 2, 64, 32, [(90, 200), (0, 300)]),
        ("bf16", 2, 1, 128, 16, [(63, 18), (64, 17), (1, 1)]), ("bf16", 4, 4, 256, 16, [(64, 40)]), ("bf16", 32, 8, 128, 64, [(128, 300)] * 5)]


def batch_of(c, lens):
    """The cache's prefixes with new tokens that its pages have no room for."""
    c.T = sum(n for _, n in lens)
    c.lens, c.start_np = lens, np.concatenate([[0], np.cumsum([n for _, n in lens])]).astype(np.int32)
    c.seq_start = torch.from_numpy(c.start_np).to(DEV)
    c.batch = c.b.KvBatch(c.seq_start, c.prefix_len, c.table, c.T, max(n for _, n in lens), None, c.status)


@gpu
@pytest.mark.parametrize("case", ROOM, ids=str)
def test_the_cache_alone_needs_no_room_for_the_block(case):
    dtype, H, Hk, D, P, lens = case
    c = Cache(dtype, H, Hk, D, P, [(p, 0) for p, _ in lens], seed=D)
    cap = c.max_pages * P
    batch_of(c, lens)
    over = [p + n > cap for p, n in lens]
    assert any(over)
    q = c.rand(c.T, H, D)
    for mask in (c.b.MRP_ATTN_CAUSAL, c.b.MRP_ATTN_BLOCK):             # (elsewhere the rule stays)
        c.status.zero_()
        out, lse = c.attend(q, mask=mask)
        assert int(c.status) == c.b.MRP_DEV_BAD_INDEX
        for (p, n), s in zip(lens, c.start_np):
            assert p + n <= cap or bool((out[s:s + n] == 7).all() and (lse[s:s + n] == 7).all())
    c.status.zero_()
    c.max_pages = 1 << 20                                          # what the plain form refuses by
    for window in (0, 50):
        for hint in (max(n for _, n in lens), 1, 10000):
            c.batch.c.max_new = hint
            out, lse = c.attend(q, mask=c.b.MRP_ATTN_PREFIX, window=window)
            close(c, q, out, lse, mask=2, window=window)
    assert int(c.status) == 0
    # a prefix that is no prefix is refused as ever
    c.max_pages = cap // P
    for bad in (cap + 1, -1, 2 ** 31 - 1):
        c.prefix_len[0] = bad
        out, lse = c.attend(q, mask=c.b.MRP_ATTN_PREFIX)
        assert int(c.status) == c.b.MRP_DEV_BAD_INDEX and (out[:lens[0][1]] == 7).all() and (lse[:lens[0][1]] == 7).all()
        c.status.zero_()


@gpu
@pytest.mark.parametrize("kind", [Cache, CacheQ8], ids=["as it is", "8 bits"])
@pytest.mark.parametrize("dtype,H,Hk,D,P,lens", [("bf16", 8, 2, 128, 16, [(64, 4), (47, 4), (0, 4)]), ("bf16", 8, 2, 128, 16, [(64, 40), (30, 3)]),
                                                 ("f32", 4, 2, 64, 16, [(64, 4), (1, 20)]), ("bf16", 4, 1, 80, 9, [(40, 30)])], ids=str)
def test_a_block_without_room_joined_with_its_own_keys(kind, dtype, H, Hk, D, P, lens):
    c = kind(dtype, H, Hk, D, P, [(p, 0) for p, _ in lens], seed=3)
    batch_of(c, lens)
    rows = c.rand(c.T, H + 2 * Hk, D)
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    out, lse = c.attend(q, mask=c.b.MRP_ATTN_PREFIX)
    c.b.mrp_packed_attention(c.ctx, c.batch, k, v, q, out, lse, mask=c.b.MRP_ATTN_BLOCK, join=True)
    r, split = half_step(dtype), 0.0 if dtype == "bf16" else 2.0 ** -20
    for b, ((p, n), s) in enumerate(zip(lens, c.start_np)):
        pages = torch.from_numpy(c.table_np[b, :-(-p // P)].astype(np.int64)).to(DEV)
        held = [pool[pages].double().permute(1, 0, 2, 3).reshape(Hk, -1, D)[:, :p] for pool in (c.k_pages, c.v_pages)]
        kk, vv = (torch.cat([h, x[s:s + n].double().transpose(0, 1)], 1).repeat_interleave(H // Hk, 0) for h, x in zip(held, (k, v)))
        x = q[s:s + n].double().transpose(0, 1)
        zz = x @ kk.transpose(1, 2) / math.sqrt(D)
        w = torch.softmax(zz, -1)
        want, reach, lw = (w @ vv).transpose(0, 1), (w @ vv.abs()).transpose(0, 1), torch.logsumexp(zz, -1).T
        size = (x.abs() @ kk.abs().transpose(1, 2) / math.sqrt(D)).amax(-1).T
        z = (D * U + split) * size + 16 * U * (size + 2) + (p + n) * U
        # one rounding of the cache's part, one of the probabilities, one of the result
        tol = reach * (4 * z + (2 * r if dtype == "bf16" else 2 * split + r))[..., None] + r * want.abs()
        assert ((out[s:s + n].double() - want).abs() <= tol).all()
        assert ((lse[s:s + n].double() - lw).abs() <= 2 * z).all()
    assert int(c.status) == 0 and TORCH[dtype] is out.dtype

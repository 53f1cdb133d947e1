"""What a workspace has to hold: packed attention on large tiles asks for more than the other calls on rows, or on pages that TMA does not
take; a workspace of their size serves those as it always did, and packed attention on tiles of 16 rows."""
import ctypes

import pytest
import torch

from test_gpu_kv import DEV, TORCH, Cache
from test_gpu_q8 import Rows

gpu = pytest.mark.gpu


def sizes(c, H, Hk, D, P, n_pages, max_pages):
    """(bytes that all calls can use, bytes of the tiles of 16 rows alone), and the geometry."""
    b = c.b
    kv = b.mrp_kv_config(H, Hk, D, P, n_pages, max_pages, 0, 0, 0, 1e4, None, 1e-6)
    least = b.mrp_config.from_buffer_copy(c.ctx.cfg)
    least.flags |= b.MRP_FLAG_FORCE_SIMT
    return tuple(int(b.lib.mrp_kv_workspace_bytes(ctypes.byref(x), ctypes.byref(kv))) for x in (c.ctx.cfg, least)), kv


def attach(c, kv, nbytes):
    """The geometry again, with `nbytes` of workspace between guards."""
    ws = torch.full((nbytes + 4096,), 0x5A, device=DEV, dtype=torch.uint8)
    off = (-ws.data_ptr()) % 256 + 1024
    torch.cuda.synchronize()
    rc = c.b.lib.mrp_kv_attach(c.ctx.handle, ctypes.byref(kv), ctypes.c_void_p(ws.data_ptr() + off), ctypes.c_size_t(nbytes))
    return rc, ws, off


def guarded(ws, off, nbytes):
    torch.cuda.synchronize()
    return bool((ws[:off] == 0x5A).all() and (ws[off + nbytes:] == 0x5A).all())


@gpu
@pytest.mark.parametrize("D,new", [(128, [300, 2, 150]), (64, [700] * 3 + [4] * 20), (256, [140, 3]), (80, [4] * 9)], ids=str)
def test_rows_in_the_workspace_of_16_row_tiles(D, new):
    H, Hk = 8, 2
    c = Rows("bf16", H, Hk, D, new, seed=D)
    (full, least), kv = sizes(c, H, Hk, D, 16, 0, 0)
    assert 0 < least < full
    rc, ws, off = attach(c, kv, least)
    assert rc == 0
    for kw in (dict(), dict(mask=1), dict(window=30, sinks=3)):
        for hint in (max(new), 1, 10000):
            c.batch.c.max_new = hint
            c.close(*c.attend(**kw), **kw)
    assert guarded(ws, off, least)
    q, out = c.q.contiguous(), torch.empty((c.T, H, D), device=DEV, dtype=TORCH["bf16"])
    c.b.mrp_qk_norm_rotate(c.ctx, None, q, None, out, None)        # (no rotation attached: the rows themselves)
    assert torch.equal(out, q)
    assert attach(c, kv, least - 1)[0] == 4
    rc, ws, off = attach(c, kv, full)
    assert rc == 0
    c.batch.c.max_new = max(new)
    c.close(*c.attend())
    assert guarded(ws, off, full)


@gpu
@pytest.mark.parametrize("dtype,P", [("bf16", 20), ("bf16", 16), ("f32", 16)])
def test_pages_in_the_workspace_they_need(dtype, P):
    H, Hk, D = 8, 2, 128
    c = Cache(dtype, H, Hk, D, P, [(700, 3), (33, 1), (0, 2), (90, 40)], seed=P)
    (full, least), kv = sizes(c, H, Hk, D, P, c.k_pages.shape[0], c.max_pages)
    need = full if dtype == "bf16" and P % 8 == 0 else least
    rc, ws, off = attach(c, kv, need)
    assert rc == 0
    q = c.rand(c.T, H, D)
    out, lse = c.attend(q)
    c.check(q, out, lse)
    rows = c.rand(c.T, 2 * Hk, D)
    own, l2 = torch.empty_like(out), torch.empty_like(lse)
    c.b.mrp_packed_attention(c.ctx, c.batch, rows[:, :Hk], rows[:, Hk:], q, own, l2)
    assert torch.isfinite(own.float()).all() and guarded(ws, off, need)
    assert attach(c, kv, need - 1)[0] == 4

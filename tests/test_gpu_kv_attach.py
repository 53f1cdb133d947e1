"""Attaching a cache geometry again, and a workspace from memory that is still in use."""
import pytest
import torch

from test_gpu_kv import Cache, DEV
from test_gpu_kv_paths import close

gpu = pytest.mark.gpu


def workspace_bytes(ctx):
    return sum(t.numel() for t in ctx.keep if t.dtype == torch.uint8)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attaching_again_takes_no_more_memory(dtype):
    c = Cache(dtype, 8, 2, 64, 16, [(900, 3), (40, 1)], seed=3)
    q = c.rand(c.T, 8, 64)
    n_pages, held, kept = c.k_pages.shape[0], workspace_bytes(c.ctx), len(c.ctx.keep)
    for more in range(1, 20):                             # a pool that grows
        c.b.mrp_kv_attach(c.ctx, 8, 2, 64, 16, n_pages + more, c.max_pages)
    assert workspace_bytes(c.ctx) == held and len(c.ctx.keep) == kept
    c.b.mrp_kv_attach(c.ctx, 8, 2, 64, 16, n_pages, c.max_pages)
    out, lse = c.attend(q)
    close(c, q, out, lse)
    assert int(c.status.item()) == 0


@gpu
def test_attaching_behind_a_call_that_still_runs():
    """The call before the attach and the one behind it, on a stream that the legacy stream does not wait for."""
    c = Cache("bf16", 32, 8, 128, 16, [(6000, 1), (2000, 1)], seed=4)
    q = c.rand(c.T, 32, 128)
    want, wl = c.attend(q)
    close(c, q, want, wl)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(10):
            out, lse = torch.full_like(want, 7.0), torch.full_like(wl, 7.0)
            torch.cuda._sleep(1000000)
            c.attend(q, out)
            c.b.mrp_kv_attach(c.ctx, 32, 8, 128, 16, c.k_pages.shape[0], c.max_pages)
            c.b.mrp_paged_attention(c.ctx, c.batch, c.k_pages, c.v_pages, q, out, lse)
            side.synchronize()
            assert torch.equal(out, want) and torch.equal(lse, wl)


@gpu
def test_a_workspace_from_memory_with_work_pending():
    """The allocator hands a block out again on its stream while a kernel there has yet to write it."""
    c = Cache("bf16", 8, 2, 128, 16, [(3000, 1)], seed=5)
    q = c.rand(c.T, 8, 128)
    size = int(c.ctx.kv_ws.numel()) if getattr(c.ctx, "kv_ws", None) is not None else c.ctx.keep[-1].numel()
    w_lm = torch.zeros((32, 64), device=DEV, dtype=torch.bfloat16)
    fresh = c.b.mrp_create(64, 64, 32, [], w_lm, max_rows=1, max_seqs=1, block_len=1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        x = torch.empty(size, dtype=torch.uint8, device=DEV)
        torch.cuda._sleep(400000000)
        x.fill_(1)
        at = x.data_ptr()
        del x
        c.b.mrp_kv_attach(fresh, 8, 2, 128, 16, c.k_pages.shape[0], c.max_pages)
        assert any(t.data_ptr() == at for t in fresh.keep)
    torch.cuda.synchronize()
    out, lse = torch.full((1, 8, 128), 7.0, device=DEV, dtype=torch.bfloat16), torch.full((1, 8), 7.0, device=DEV)
    c.b.mrp_paged_attention(fresh, c.batch, c.k_pages, c.v_pages, q, out, lse)
    close(c, q, out, lse)

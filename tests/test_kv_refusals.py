"""Arguments of the paged-cache calls that the host refuses beside those of test_gpu_kv_paths.py."""
import ctypes

import pytest


def workspace_bytes(**kw):
    from paper_2605_18817_b200 import binding as b
    cfg = b.mrp_config(64, 64, 32, 0, 1, 4, 1, b.MRP_BF16, 1e-6, 0, 0)
    a = dict(n_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10, max_pages=4, page_stride=0, rot_dim=128, rot_interleaved=0,
             rot_theta=1e4, inv_freq=None, norm_eps=1e-6)
    a.update(kw)
    return int(b.lib.mrp_kv_workspace_bytes(ctypes.byref(cfg), ctypes.byref(b.mrp_kv_config(*a.values()))))


def test_numbers_of_a_geometry_that_are_not_finite():
    assert workspace_bytes() > 0 and workspace_bytes(rot_theta=1e-300) > 0 and workspace_bytes(norm_eps=0.0) > 0
    for kw in (dict(rot_theta=5e-324), dict(norm_eps=float("inf")), dict(rot_theta=float("nan")),
               dict(inv_freq=(ctypes.c_double * 64)(*([0.5] * 63 + [float("nan")])))):
        assert workspace_bytes(**kw) == 0, kw


@pytest.mark.gpu
def test_a_scale_beyond_fp32_in_base_2():
    from test_gpu_kv import Cache
    c = Cache("bf16", 4, 2, 128, 16, [(20, 3)], seed=1)
    q = c.rand(3, 4, 128)
    with pytest.raises(c.b.MrpError) as e:
        c.attend(q, scale=3e38)
    assert e.value.status == 1
    c.attend(q, scale=2e38)
    out, lse = c.attend(q)
    c.check(q, out, lse)


def test_pools_whose_dimensions_of_one_entry_have_other_strides():
    """One key head stored [pages, rows, 1, features], one row a page, one page: the same memory, other strides by name."""
    import torch
    from types import SimpleNamespace
    from paper_2605_18817_b200 import binding as b

    def shape(n, hk, p, d):
        return b._KvShape(torch.float32, -1, (2 * hk, d), (hk, d), (n, hk, p, d), (hk * p * d, p * d, d, 1), 4)
    batch = SimpleNamespace(max_pages=4, device=-1)
    for n, hk, p, pool in ((6, 1, 16, torch.zeros(6, 16, 1, 8).transpose(1, 2)), (6, 3, 1, torch.zeros(6, 1, 3, 8).transpose(1, 2)),
                           (1, 3, 16, torch.zeros(3, 1, 16, 8).transpose(0, 1)), (6, 3, 16, torch.zeros(6, 3, 16, 8))):
        got = b._pools(shape(n, hk, p, 8), batch, pool, pool)
        assert got.k == got.v == pool.data_ptr()
    for n, hk, p, pool in ((6, 2, 16, torch.zeros(6, 16, 2, 8).transpose(1, 2)), (6, 1, 16, torch.zeros(6, 1, 16, 16)[..., :8]),
                           (6, 1, 16, torch.zeros(12, 1, 16, 8)[::2])):
        with pytest.raises(ValueError):
            b._pools(shape(n, hk, p, 8), batch, pool, pool)

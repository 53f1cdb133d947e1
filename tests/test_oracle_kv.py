"""The 64-bit statements of the paged-cache operators (oracle/kv.py) against closed forms and library restatements."""
import math

import numpy as np
import pytest
import torch

from oracle import kv


def cache(lens, H=4, Hk=2, D=8, P=5, seed=0):
    rng = np.random.default_rng(seed)
    need = [-(-max(1, p + n) // P) for p, n in lens]
    table = np.full((len(lens), max(need)), -1, np.int32)
    ids = list(rng.permutation(sum(need)))
    for b, c in enumerate(need):
        table[b, :c] = [ids.pop() for _ in range(c)]
    pools = [rng.standard_normal((sum(need), Hk, P, D)) for _ in range(2)]
    start = np.concatenate([[0], np.cumsum([n for _, n in lens])])
    q = rng.standard_normal((int(start[-1]), H, D))
    return q, pools[0], pools[1], start, np.array([p for p, _ in lens]), table, P


@pytest.mark.parametrize("mask", [kv.CAUSAL, kv.BLOCK, kv.PREFIX])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0), (4, 2), (1, 1)])
def test_attention_is_the_masked_softmax(mask, window, sinks):
    lens = [(7, 3), (0, 4), (12, 1), (3, 0)]
    args = cache(lens)
    q, kp, vp, start, pre, table, P = args
    out, lse, reach, size = kv.attention(*args, mask, window, sinks)
    for b, (p, n) in enumerate(lens):
        length = p + n
        k, v = (torch.from_numpy(np.stack([pool[table[b, j // P], :, j % P] for j in range(length)], 1)) if length else None for pool in (kp, vp))
        for i in range(n):
            for h in range(q.shape[1]):
                z = k[h // 2] @ torch.from_numpy(q[start[b] + i, h]) / math.sqrt(q.shape[2])
                j = torch.arange(length)
                hidden = {kv.CAUSAL: j > p + i, kv.BLOCK: j < 0, kv.PREFIX: j >= p}[mask]
                if window:
                    hidden |= (j <= p + i - window) & (j >= sinks)
                z[hidden] = -math.inf
                if hidden.all():
                    assert (out[start[b] + i, h] == 0).all() and lse[start[b] + i, h] == -math.inf
                    continue
                w = torch.softmax(z, 0)
                np.testing.assert_allclose(out[start[b] + i, h], (w @ v[h // 2]).numpy(), atol=1e-12)
                np.testing.assert_allclose(lse[start[b] + i, h], torch.logsumexp(z, 0).item(), atol=1e-12)
                assert (reach[start[b] + i, h] >= np.abs(out[start[b] + i, h]) - 1e-12).all() and size[start[b] + i, h] >= z.max() - 1e-12


def test_equal_keys_average_the_values_and_scale_the_log_sum():
    q, kp, vp, start, pre, table, P = cache([(9, 2)])
    kp[:] = 0.25
    out, lse, _, _ = kv.attention(q, kp, vp, start, pre, table, P, kv.CAUSAL, scale=2.0)
    v = kv.gather(vp, table, 0, 11, P)
    for i in range(2):
        np.testing.assert_allclose(out[i], np.repeat(v[:, :10 + i].mean(1), 2, 0), atol=1e-12)
        np.testing.assert_allclose(lse[i], 2.0 * 0.25 * q[i].sum(-1) + math.log(10 + i), atol=1e-12)


def test_two_passes_join_by_their_log_sums():
    args = cache([(11, 4), (2, 3)])
    whole, lw, _, _ = kv.attention(*args, kv.CAUSAL)
    a, la, _, _ = kv.attention(*args, kv.CAUSAL, window=3)
    lo, ll = np.zeros_like(whole), np.zeros_like(lw)
    q, kp, vp, start, pre, table, P = args
    for b in range(2):                                    # what the window leaves out, as a pass of its own
        for i in range(start[b + 1] - start[b]):
            r = start[b] + i
            n = max(0, pre[b] + i + 1 - 3)
            k, v = kv.gather(kp, table, b, n, P), kv.gather(vp, table, b, n, P)
            for h in range(q.shape[1]):
                z = k[h // 2] @ q[r, h] / math.sqrt(q.shape[2])
                ll[r, h] = np.log(np.exp(z).sum()) if n else -np.inf
                lo[r, h] = np.exp(z) @ v[h // 2] / np.exp(z).sum() if n else 0
    wa, wl = np.exp(la - lw)[..., None], np.exp(ll - lw)[..., None]
    np.testing.assert_allclose(a * wa + lo * wl, whole, atol=1e-12)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_depends_on_distance_alone(interleaved):
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((1, 2, 12)), rng.standard_normal((1, 2, 12))
    rot = lambda z, p: kv.norm_rotate(z, [p], None, 8, 100.0, None, interleaved)      # noqa: E731
    np.testing.assert_allclose(np.linalg.norm(rot(x, 37), axis=-1), np.linalg.norm(x, axis=-1), atol=1e-12)
    np.testing.assert_allclose((rot(x, 5) * rot(y, 3)).sum(-1), (rot(x, 1005) * rot(y, 1003)).sum(-1), atol=1e-11)
    np.testing.assert_allclose(rot(x, 0), x, atol=0)
    np.testing.assert_allclose(rot(x, 9)[..., 8:], x[..., 8:], atol=0)
    np.testing.assert_allclose(rot(rot(x, 4), -4), x, atol=1e-12)
    np.testing.assert_allclose(rot(x, 2), kv.norm_rotate(x, [2], None, 8, 1.0, [100.0 ** (-j / 4) for j in range(4)], interleaved), atol=1e-12)


def test_norm_is_unit_root_mean_square_times_gamma():
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((3, 2, 16)) * 5, rng.standard_normal(16)
    y = kv.norm_rotate(x, [0, 0, 0], g, eps=0.0)
    np.testing.assert_allclose(np.sqrt((y / g) ** 2).mean(-1).shape, (3, 2))
    np.testing.assert_allclose(((y / g) ** 2).mean(-1), 1.0, atol=1e-12)


def test_append_stores_rows_where_attention_finds_them():
    lens = [(4, 3), (0, 2), (6, 0)]
    q, kp, vp, start, pre, table, P = cache(lens)
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    kn, vn = kv.append(kp, vp, k, v, start, pre, table, P)
    for b, (p, n) in enumerate(lens):
        got, old = kv.gather(kn, table, b, p + n, P), kv.gather(kp, table, b, p + n, P)
        assert np.array_equal(got[:, :p], old[:, :p])
        assert np.array_equal(got[:, p:], k[start[b]:start[b] + n].transpose(1, 0, 2))
    assert (kn != kp).any(-1).sum() == 5 * 2 and (vn != vp).any(-1).sum() == 5 * 2
    # a page outside the pool takes nothing and reads as zeros; a sequence that does not fit is skipped
    bad = table.copy()
    bad[0, 0] = 99
    kb, _ = kv.append(kp, vp, k, v, start, pre, bad, P)
    assert np.array_equal(kv.gather(kb, bad, 0, 5, P), np.zeros((2, 5, 8)))
    assert [b for b, *_ in kv.sequences([0, 3, 2, 9, 9], [0, 0, 0, 99], 5, 20)] == [0]

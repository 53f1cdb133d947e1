"""Probabilities as two bf16 parts: where a sequence has up to 16 rows (new tokens times query heads of a key head), whatever
the other sequences of the batch and whatever the host believes of their lengths, and on 16-row tiles for all rows.

What tells two parts from one: keys in pairs with nearly the same score and opposite values, so the output is small beside
sum p |v| and the rounding of the probabilities is most of it.  The tolerance is that of test_gpu_kv.py with 2^-16 (two
parts leave out 2^-17 of a probability; twice that, as there) in the place of bf16's 2^-8; the statement with probabilities
rounded to bf16 once has to miss it."""
import math

import numpy as np
import pytest
import torch

from oracle import kv as ref
from test_gpu_kv import DEV, U, Cache, f64

gpu = pytest.mark.gpu


def paired(c):
    """Keys 2 m and 2 m + 1 of every sequence: the second 1 + 2^-6 times the first, its value the first's with the other sign."""
    for b, (p, n) in enumerate(c.lens):
        k, v = c.rand(p + n, c.Hk, c.D), c.rand(p + n, c.Hk, c.D)
        k[1::2] = (k[0::2].float() * (1 + 2.0 ** -6)).to(k.dtype)[:k[1::2].shape[0]]
        v[1::2] = -v[0::2][:v[1::2].shape[0]]
        for j in range(p + n):
            c.k_pages[c.table_np[b, j // c.P], :, j % c.P], c.v_pages[c.table_np[b, j // c.P], :, j % c.P] = k[j], v[j]


def bounds(c, q, sequences):
    """(rows, output, tolerance, output with probabilities rounded to bf16 once) of the tokens of `sequences`."""
    rows, out, tol, once = [], [], [], []
    g = c.H // c.Hk
    for b, s, n, p in ref.sequences(c.start_np, c.pre_np, c.T, c.max_pages * c.P):
        if b not in sequences:
            continue
        k, v = (ref.gather(f64(x), c.table_np, b, p + n, c.P) for x in (c.k_pages, c.v_pages))
        for i in range(n):
            x = f64(q[s + i])
            kk, vv = np.repeat(k[:, :p + i + 1], g, 0), np.repeat(v[:, :p + i + 1], g, 0)
            z = np.einsum("hd,hjd->hj", x, kk) / math.sqrt(c.D)
            e = np.exp(z - z.max(-1, keepdims=True))
            total = e.sum(-1, keepdims=True)
            o, reach = np.einsum("hj,hjd->hd", e, vv) / total, np.einsum("hj,hjd->hd", e, np.abs(vv)) / total
            size = (np.einsum("hd,hjd->hj", np.abs(x), np.abs(kk)) / math.sqrt(c.D)).max(-1)
            zt = c.D * U * size + 4 * U * (size + 1)
            rows.append(s + i)
            out.append(o)
            tol.append(reach * (2 * zt + 2 * (p + n + 1) * U + 2.0 ** -16)[:, None] + 2.0 ** -8 * np.abs(o) + 1e-30)
            h = torch.from_numpy(e).to(torch.bfloat16).double().numpy()
            once.append(np.einsum("hj,hjd->hd", h, vv) / total)
    return (np.array(x) for x in (rows, out, tol, once))


def check(c, q, out, sequences):
    rows, want, tol, once = bounds(c, q, sequences)
    assert (np.abs(once - want) > tol).any()               # (one part would show)
    got = f64(out)[rows]
    worst = (np.abs(got - want) / tol).max()
    assert worst <= 1.0, worst


TWO = [
    # H, Hk, D, P, lens, sequences of up to 16 rows
    (4, 2, 64, 16, [(21, 2), (60, 8)], [0, 1]),                          # a batch of such sequences alone
    (8, 2, 128, 16, [(21, 1), (39, 4)], [0, 1]),
    (4, 1, 64, 32, [(900, 3)], [0]),                                     # cut in pieces
    (8, 2, 256, 16, [(21, 1), (39, 4)], [0, 1]),
    (8, 2, 64, 16, [(21, 1), (300, 40), (39, 4)], [0, 2]),               # beside one of more rows
    (8, 2, 128, 16, [(21, 1), (300, 20), (39, 4), (30, 2)], [0, 2, 3]),
    (8, 2, 128, 64, [(21, 1), (2500, 10), (900, 1)], [0, 2]),
    (8, 2, 256, 32, [(21, 1), (300, 20), (39, 4), (30, 2)], [0, 2, 3]),
    (15, 5, 80, 24, [(21, 1), (300, 20), (39, 5), (30, 2)], [0, 2, 3]),
    (64, 8, 64, 32, [(21, 1)] + [(300, 20)] * 20 + [(39, 2)], [0, 21]),  # beside many
    (64, 8, 128, 32, [(21, 1)] + [(300, 20)] * 20 + [(39, 2)], [0, 21]),
    (32, 8, 128, 32, [(21, 1), (0, 1300), (39, 4)], [0, 2]),             # beside a prompt
]


@gpu
@pytest.mark.parametrize("case", TWO, ids=lambda c: "H%d-%d-D%d-P%d-n%d" % (c[0], c[1], c[2], c[3], len(c[4])))
def test_sequences_of_up_to_16_rows(case):
    H, Hk, D, P, lens, short = case
    c = Cache("bf16", H, Hk, D, P, lens, seed=H + D)
    paired(c)
    q = c.rand(c.T, H, D) * 1.5
    for hint in (c.batch.c.max_new, 1, 17, 10000):
        c.batch.c.max_new = hint
        out, _ = c.attend(q)
        check(c, q, out, short)
    assert int(c.status.item()) == 0


@gpu
@pytest.mark.parametrize("H,Hk,D,P", [(4, 2, 64, 16), (8, 2, 128, 20), (3, 1, 256, 16)])
def test_tiles_of_16_rows(H, Hk, D, P):
    lens = [(21, 2), (39, 9), (30, 20)]
    c = Cache("bf16", H, Hk, D, P, lens, seed=D)
    paired(c)
    q = c.rand(c.T, H, D) * 1.5
    w_lm = torch.zeros((32, 64), device=DEV, dtype=torch.bfloat16)
    other = c.b.mrp_create(64, 64, 32, [], w_lm, max_rows=1, max_seqs=3, block_len=1, flags=c.b.MRP_FLAG_FORCE_SIMT)
    c.b.mrp_kv_attach(other, H, Hk, D, P, c.k_pages.shape[0], c.max_pages)
    out = torch.empty_like(q)
    c.b.mrp_paged_attention(other, c.batch, c.k_pages, c.v_pages, q, out)
    check(c, q, out, [0, 1, 2])

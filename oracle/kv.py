"""Plain 64-bit statements of the paged-cache operators (per-head norm and rotation, append, attention), in numpy, one
sequence and one head at a time.  Test infrastructure only."""
import math

import numpy as np

CAUSAL, BLOCK, PREFIX = 0, 1, 2


def norm_rotate(x, positions, gamma=None, rot=0, theta=10000.0, inv_freq=None, interleaved=False, eps=1e-6):
    """x [T, heads, D] -> float64: x * rsqrt(mean(x^2) + eps) * gamma (with gamma), then pair j of the first `rot` features
    turned by positions[t] * w_j."""
    y = np.array(x, dtype=np.float64)
    if gamma is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(gamma, np.float64)
    out = y.copy()
    for j in range(rot // 2):
        w = inv_freq[j] if inv_freq is not None else theta ** (-2.0 * j / rot)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        for t in range(y.shape[0]):
            c, s = math.cos(float(positions[t]) * w), math.sin(float(positions[t]) * w)
            out[t, :, a] = y[t, :, a] * c - y[t, :, b] * s
            out[t, :, b] = y[t, :, b] * c + y[t, :, a] * s
    return out


def sequences(seq_start, prefix_len, n_tokens, cap):
    """(b, first row, new tokens, cached positions) of the sequences that fit."""
    for b in range(len(prefix_len)):
        s, e, p = int(seq_start[b]), int(seq_start[b + 1]), int(prefix_len[b])
        if 0 <= s <= e <= n_tokens and 0 <= p and p + e - s <= cap:
            yield b, s, e - s, p


def append(k_pages, v_pages, k, v, seq_start, prefix_len, page_table, page_size):
    """Copies of the pools [n_pages, Hk, P, D] with the rows k, v [T, Hk, D] (already normalised and rotated) stored."""
    kp, vp = np.array(k_pages, np.float64), np.array(v_pages, np.float64)
    for b, s, n, p in sequences(seq_start, prefix_len, k.shape[0], page_table.shape[1] * page_size):
        for i in range(n):
            page = page_table[b, (p + i) // page_size]
            if 0 <= page < kp.shape[0]:
                kp[page, :, (p + i) % page_size] = k[s + i]
                vp[page, :, (p + i) % page_size] = v[s + i]
    return kp, vp


def visible(mask, prefix, new, i, window, sinks):
    """Positions that the new token at place i sees, ascending."""
    pos = prefix + i
    end = {CAUSAL: pos + 1, BLOCK: prefix + new, PREFIX: prefix}[mask]
    return [j for j in range(end) if window <= 0 or j > pos - window or j < sinks]


def gather(pages, page_table, b, length, page_size):
    """[Hk, length, D] float64 rows of sequence b; pages outside the pool read as zeros."""
    out = np.zeros((pages.shape[1], length, pages.shape[3]))
    for j in range(length):
        page = page_table[b, j // page_size]
        if 0 <= page < pages.shape[0]:
            out[:, j] = pages[page, :, j % page_size]
    return out


def attention(q, k_pages, v_pages, seq_start, prefix_len, page_table, page_size, mask=CAUSAL, window=0, sinks=0, scale=0.0,
              out=None):
    """(out [T, H, D], lse [T, H], reach [T, H, D], size [T, H]) in float64; rows of no sequence keep `out` (zeros) and
    lse 0.  reach = sum_j p_j |v_j| and size = max_j scale sum |q||k_j| are what rounding errors are measured against."""
    T, H, D = q.shape
    Hk = k_pages.shape[1]
    g = H // Hk
    scale = scale or 1.0 / math.sqrt(D)
    o = np.zeros((T, H, D)) if out is None else np.array(out, np.float64)
    lse, reach, size = np.zeros((T, H)), np.zeros((T, H, D)), np.zeros((T, H))
    for b, s, n, p in sequences(seq_start, prefix_len, T, page_table.shape[1] * page_size):
        length = p + n if mask != PREFIX else p
        k = gather(k_pages, page_table, b, length, page_size)
        v = gather(v_pages, page_table, b, length, page_size)
        for i in range(n):
            seen = np.array(visible(mask, p, n, i, window, sinks), dtype=np.int64)
            for h in range(H):
                if seen.size == 0:
                    o[s + i, h], lse[s + i, h] = 0.0, -np.inf
                    continue
                kk, vv = k[h // g][seen], v[h // g][seen]
                x = np.asarray(q[s + i, h], np.float64)
                z = kk @ x * scale
                m = z.max()
                e = np.exp(z - m)
                o[s + i, h] = e @ vv / e.sum()
                lse[s + i, h] = m + math.log(e.sum())
                reach[s + i, h] = e @ np.abs(vv) / e.sum()
                size[s + i, h] = (np.abs(kk) @ np.abs(x)).max() * abs(scale)
    return o, lse, reach, size


# ---- the cache in 8 bits (codes: oracle/fp8.py) ------------------------------------------------------------------------

def q8_rows(x):
    """Rows x [.., D] -> (e4m3 codes uint8 [.., D], scale bytes uint8 [..]): row = codes * 2^(byte - 127), the exponent the
    smallest one >= -127 with max |row| <= 448 * 2^E, 0 for a row of zeros, codes of rows with E = 120 at most 240; byte 255 (codes 0) where a value is not finite."""
    from oracle import fp8
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, x.shape[-1])
    bad = ~np.isfinite(flat).all(-1)
    flat = np.where(bad[:, None], 0.0, flat)
    scale = np.maximum(fp8.row_scales(flat), 2.0 ** -127)
    top = np.where(scale == 2.0 ** 120, 240.0, 448.0)[:, None]             # (256 * 2^120 is infinite in fp32 and bf16)
    codes = fp8.encode(np.clip(flat / scale[:, None], -top, top))
    byte = np.where(bad, 255, np.frexp(scale)[1] - 1 + 127).astype(np.uint8)
    return codes.reshape(x.shape), byte.reshape(x.shape[:-1])


def q8_values(codes, byte):
    """What codes and scale bytes stand for, float64: NaN codes and rows of byte 255 are NaN."""
    from oracle import fp8
    codes, byte = np.asarray(codes, np.uint8), np.asarray(byte, np.uint8)
    v = np.where((codes & 0x7F) == 0x7F, np.nan, fp8.decode(codes)) * 2.0 ** (byte.astype(np.float64) - 127)[..., None]
    return np.where((byte == 255)[..., None], np.nan, v)


def join(o1, l1, o2, l2):
    """Two passes over disjoint sets of keys, as one: (out, lse)."""
    l = np.logaddexp(l1, l2)
    with np.errstate(invalid="ignore"):
        w1, w2 = (np.where(np.isneginf(x), 0.0, np.exp(x - l)) for x in (l1, l2))
    return np.where(w1[..., None] > 0, w1[..., None] * o1, 0.0) + np.where(w2[..., None] > 0, w2[..., None] * o2, 0.0), l


def packed(q, k, v, seq_start, mask=CAUSAL, window=0, sinks=0, scale=0.0):
    """Attention of rows over each other: every sequence is a cache of its own rows, all of them new."""
    n_seqs = len(seq_start) - 1
    longest = max([1] + [int(seq_start[b + 1]) - int(seq_start[b]) for b in range(n_seqs)])
    kp, vp = (np.zeros((n_seqs, k.shape[1], longest, k.shape[2])) for _ in range(2))
    for b in range(n_seqs):
        s, e = int(seq_start[b]), int(seq_start[b + 1])
        if 0 <= s <= e <= q.shape[0]:
            kp[b, :, :e - s], vp[b, :, :e - s] = np.swapaxes(k[s:e], 0, 1), np.swapaxes(v[s:e], 0, 1)
    return attention(q, kp, vp, seq_start, np.zeros(n_seqs, np.int32), np.arange(n_seqs)[:, None], longest, mask, window, sinks, scale)

"""The attention of a block behind its paged key / value cache, operator by operator: cases, inputs, plain forms, work.

Three operators that one layer of a serving step runs in this order:
  rotate   RMSNorm of every query and key head and the rotation by its position, in one pass (mrp_qk_norm_rotate)
  append   the same for the step's keys (and queries), keys and values stored in the pages of their sequences (mrp_kv_append)
  attend   the step's queries over the pages: causal, block or prefix mask, window and first tokens (mrp_paged_attention)

`own` false: elementary torch operations in 32 bits (angles in 64), rounded once at the end.  `own` true: the library's calls.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA = 1.0e6
EPS = 1.0e-6
CAUSAL, BLOCK, PREFIX = 0, 1, 2
MASKS = {"causal": CAUSAL, "block": BLOCK, "prefix": PREFIX}


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one block of 4 positions of one sequence at the decode shape (d = 2048: 16 heads of 128): latency
        dict(name="rotate block of 4", op="rotate", dtype="bf16", tokens=4, heads=16, kv_heads=8, dim=128, rot=128,
             interleaved=False, norm=True, far=40000),
        # a long prompt of the d = 4096 shape, rows of the packed projection output
        dict(name="rotate prompt", op="rotate", dtype="bf16", tokens=16384, heads=32, kv_heads=8, dim=128, rot=128,
             interleaved=False, norm=True, far=16384),
        # 32-bit, half of the features rotated in adjacent pairs, far positions, an odd number of tokens
        dict(name="rotate f32 far", op="rotate", dtype="f32", tokens=1021, heads=12, kv_heads=4, dim=80, rot=40,
             interleaved=True, norm=False, far=1 << 20),
        # a serving step: 32 sequences, blocks of 4 positions
        dict(name="append blocks", op="append", dtype="bf16", seqs=32, new_lo=4, new_hi=4, pre_lo=100, pre_hi=9000,
             heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, norm=True, page=16, mix=1),
        # ragged prompts entering the cache
        dict(name="append prompts", op="append", dtype="bf16", seqs=9, new_lo=300, new_hi=3900, pre_lo=0, pre_hi=2000,
             heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, norm=True, page=64, mix=2),
        # one new token of one sequence: latency
        dict(name="attend one token", op="attend", dtype="bf16", seqs=1, new_lo=1, new_hi=1, pre_lo=2047, pre_hi=2047,
             heads=16, kv_heads=8, dim=128, page=16, mask="causal", window=0, sinks=0, mix=3),
        # one token each of 64 ragged sequences
        dict(name="attend 64 ragged", op="attend", dtype="bf16", seqs=64, new_lo=1, new_hi=1, pre_lo=16, pre_hi=8191,
             heads=32, kv_heads=8, dim=128, page=64, mask="causal", window=0, sinks=0, mix=4),
        # active blocks of 16 that see themselves whole
        dict(name="attend blocks of 16", op="attend", dtype="bf16", seqs=24, new_lo=16, new_hi=16, pre_lo=200, pre_hi=6000,
             heads=32, kv_heads=8, dim=128, page=32, mask="block", window=0, sinks=0, mix=5),
        # long caches read through a window, the first tokens kept
        dict(name="attend window", op="attend", dtype="bf16", seqs=12, new_lo=4, new_hi=4, pre_lo=20000, pre_hi=60000,
             heads=32, kv_heads=8, dim=128, page=16, mask="causal", window=4096, sinks=100, mix=6),
        # a chunk of two prompts behind what is cached already
        dict(name="attend prompt chunk", op="attend", dtype="bf16", seqs=2, new_lo=1900, new_hi=2100, pre_lo=5000, pre_hi=6200,
             heads=32, kv_heads=8, dim=128, page=64, mask="causal", window=0, sinks=0, mix=7),
        # a mixed step, odd sizes everywhere: single tokens beside short prompts, three heads a key head, pages of 24
        dict(name="attend mixed odd", op="attend", dtype="bf16", seqs=13, new_lo=1, new_hi=150, pre_lo=0, pre_hi=1500,
             heads=15, kv_heads=5, dim=80, page=24, mask="causal", window=0, sinks=0, mix=8),
        # 32-bit cache, the prefix alone (the block's own keys are another pass's), a head of its own for every query head
        dict(name="attend f32 prefix", op="attend", dtype="f32", seqs=6, new_lo=4, new_hi=4, pre_lo=0, pre_hi=4096,
             heads=16, kv_heads=16, dim=64, page=128, mask="prefix", window=0, sinks=0, mix=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "append", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 4, 5, 8, 16])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 8) if kv * g <= 32])
    dim = rng.choice([64, 128, 128, rng.randrange(4, 33) * 8])
    if op == "rotate":
        return dict(op=op, dtype=dtype, tokens=_log(rng, 1, 12000 if dim <= 128 else 6000), heads=heads, kv_heads=kv, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, 20]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.7, far=_log(rng, 64, 1 << 20))
    seqs = _log(rng, 1, 48)
    page = rng.choice([16, 32, 64, 128, rng.randrange(5, 200)])
    if op == "append":
        hi = min(_log(rng, 1, 4000), (16000 if dim <= 128 else 8000) // seqs)
        return dict(op=op, dtype=dtype, seqs=seqs, new_lo=rng.randrange(0, hi + 1), new_hi=hi, pre_lo=0, pre_hi=_log(rng, 1, 2000),
                    heads=heads, kv_heads=kv, dim=dim, rot=rng.choice([dim, dim // 2]), interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.7, page=page, mix=rng.randrange(1 << 20))
    long = min(_log(rng, 16, 30000), 110000 // seqs)
    new = min(_log(rng, 1, 700), 6000 // seqs)
    new = 1 if rng.random() < 0.3 else new if new * seqs * long < 2e7 else max(1, int(2e7 / (seqs * long)))
    if dtype == "f32" or dim > 128:
        long, new = min(long, 30000 // seqs), min(new, 300)
    window = rng.choice([0, 0, _log(rng, 1, 4096)])
    return dict(op=op, dtype=dtype, seqs=seqs, new_lo=1 if rng.random() < 0.5 else new, new_hi=new, pre_lo=rng.randrange(0, long),
                pre_hi=long, heads=heads, kv_heads=kv, dim=dim, page=page, mask=rng.choice(["causal", "causal", "block", "prefix"]),
                window=window, sinks=rng.choice([0, 4, 77]) if window else 0, mix=rng.randrange(1 << 20))


def _lengths(case):
    """(cached tokens, new tokens) of every sequence: part of the case, not of the seed."""
    r = random.Random(case["mix"])
    pre = [r.randint(case["pre_lo"], case["pre_hi"]) for _ in range(case["seqs"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    pre[-1], new[0] = case["pre_hi"], case["new_hi"]
    return pre, new


# ---- inputs --------------------------------------------------------------------------------------------------------

_contexts = {}


def _context(dev, dtype, seqs, shape):
    """One library context per geometry, as a program keeps one per model."""
    from paper_2605_18817_b200 import binding
    key = (str(dev), dtype, seqs, tuple(sorted(shape.items())))
    if key not in _contexts:
        w_lm = torch.zeros((32, 64), device=dev, dtype=DTYPES[dtype])
        ctx = binding.mrp_create(64, 64, 32, [], w_lm, max_rows=1, max_seqs=seqs, block_len=1)
        binding.mrp_kv_attach(ctx, **shape)
        _contexts[key] = ctx
    return _contexts[key]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    s = dict(case=case)
    if case["op"] == "rotate":
        T = case["tokens"]
        # the rows of a packed projection output: queries, keys, values of a token side by side
        s["qkv"] = normal(T, (H + 2 * Hk) * D)
        s["positions"] = torch.randint(0, case["far"], (T,), generator=g, device=dev, dtype=torch.int32)
    else:
        pre, new = _lengths(case)
        B, T, P = case["seqs"], sum(new), case["page"]
        total = [p + n for p, n in zip(pre, new)]
        per = max(1, max(-(-t // P) for t in total))
        used = sum(-(-t // P) for t in total)
        n_pages = used + 3
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        counts = torch.tensor([-(-t // P) for t in total], device=dev)
        col = torch.arange(per, device=dev)
        first = counts.cumsum(0) - counts
        slot = first[:, None] + torch.minimum(col[None], (counts[:, None] - 1).clamp(min=0))
        s["page_table"] = order[slot.clamp(max=n_pages - 1)].contiguous()
        s["prefix_len"] = torch.tensor(pre, device=dev, dtype=torch.int32)
        s["seq_start"] = torch.tensor([0] + list(torch.tensor(new).cumsum(0).tolist()), device=dev, dtype=torch.int32)
        s["k_pages"] = normal(n_pages, Hk, P, D)
        s["v_pages"] = normal(n_pages, Hk, P, D)
        s["longest"], s["most_new"], s["n_tokens"] = max(total), max(max(new), 1), T
        s["qkv"] = normal(T, (H + 2 * Hk) * D)
        if case["op"] == "attend":
            s["qkv"] *= 1.5                     # scores spread like those of trained heads
    T = s["qkv"].shape[0]
    rows = s["qkv"].view(T, H + 2 * Hk, D)
    s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    if case.get("norm"):
        s["gamma_q"], s["gamma_k"] = 1 + 0.1 * normal(D), 1 + 0.1 * normal(D)
    s["q_out"] = torch.zeros((T, H, D), device=dev, dtype=dt)
    s["k_out"] = torch.zeros((T, Hk, D), device=dev, dtype=dt)
    s["lse"] = torch.zeros((T, H), device=dev, dtype=torch.float32)
    if own:
        from paper_2605_18817_b200 import binding
        shape = dict(n_heads=H, n_kv_heads=Hk, head_dim=D, page_size=case.get("page", 16), rot_dim=case.get("rot", 0),
                     rot_theta=THETA, rot_interleaved=bool(case.get("interleaved")), norm_eps=EPS)
        if "page_table" in s:
            shape.update(n_pages=s["k_pages"].shape[0], max_pages=s["page_table"].shape[1])
        s["ctx"] = _context(dev, case["dtype"], case.get("seqs", 1), shape)
        if "page_table" in s:
            s["batch"] = binding.KvBatch(s["seq_start"], s["prefix_len"], s["page_table"], s["n_tokens"], s["most_new"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"rotate": _rotate, "append": _append, "attend": _attend}[case["op"]](s, case)


def _run_own(s, case):
    from paper_2605_18817_b200 import binding
    gq, gk = s.get("gamma_q"), s.get("gamma_k")
    if case["op"] == "rotate":
        binding.mrp_qk_norm_rotate(s["ctx"], s["positions"], s["q"], s["k"], s["q_out"], s["k_out"], gq, gk)
        return s["q_out"], s["k_out"]
    if case["op"] == "append":
        binding.mrp_kv_append(s["ctx"], s["batch"], s["k_pages"], s["v_pages"], s["k"], s["v"], gk, s["q"], s["q_out"], gq)
        return s["q_out"], s["k_pages"], s["v_pages"]
    binding.mrp_paged_attention(s["ctx"], s["batch"], s["k_pages"], s["v_pages"], s["q"], s["q_out"], s["lse"],
                                mask=MASKS[case["mask"]], window=case["window"], sinks=case["sinks"])
    return s["q_out"], s["lse"]


def _norm_rotate(x, gamma, positions, case):
    """x [T, heads, D] in its type -> 32 bits: RMSNorm over D, then the first `rot` features turned by their angles."""
    x = x.float()
    if gamma is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.float()
    rot = case["rot"]
    if rot == 0:
        return x
    j = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    angle = positions.double()[:, None] * THETA ** (-2.0 * j / rot)
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * c - b * n, b * c + a * n
    turned = torch.stack((u, w), -1).flatten(-2) if case["interleaved"] else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _rotate(s, case):
    dt = s["q"].dtype
    return (_norm_rotate(s["q"], s.get("gamma_q"), s["positions"], case).to(dt),
            _norm_rotate(s["k"], s.get("gamma_k"), s["positions"], case).to(dt))


def _places(s):
    """Of every token: its sequence, its place among the sequence's new tokens, its position."""
    t = torch.arange(s["qkv"].shape[0], device=s["qkv"].device)
    b = torch.searchsorted(s["seq_start"][1:].long(), t, right=True)
    i = t - s["seq_start"].long()[b]
    return b, i, s["prefix_len"].long()[b] + i


def _append(s, case):
    b, _, pos = _places(s)
    page, row = s["page_table"].long()[b, pos // case["page"]], pos % case["page"]
    dt = s["k"].dtype
    s["k_pages"][page, :, row] = _norm_rotate(s["k"], s.get("gamma_k"), pos, case).to(dt)
    s["v_pages"][page, :, row] = s["v"]
    return _norm_rotate(s["q"], s.get("gamma_q"), pos, case).to(dt), s["k_pages"], s["v_pages"]


def _attend(s, case):
    dev, dt = s["q"].device, s["q"].dtype
    H, Hk, D, P = case["heads"], case["kv_heads"], case["dim"], case["page"]
    B, N, S, T = case["seqs"], s["most_new"], s["longest"], s["q"].shape[0]
    start, pre = s["seq_start"].long(), s["prefix_len"].long()
    n = start[1:] - start[:-1]
    j = torch.arange(S, device=dev)
    page = s["page_table"].long()[:, j // P]
    in_use = (j[None] < (pre + n)[:, None])[:, :, None, None]
    k = s["k_pages"][page, :, j % P].float().masked_fill(~in_use, 0.0)      # [B, S, Hk, D]
    v = s["v_pages"][page, :, j % P].float().masked_fill(~in_use, 0.0)
    i = torch.arange(N, device=dev)
    q = s["q"][(start[:-1, None] + i[None]).clamp(max=T - 1)].float().view(B, N, Hk, H // Hk, D)
    z = torch.einsum("bnhgd,bshd->bhgns", q, k) * (1.0 / math.sqrt(D))
    pos = pre[:, None] + i[None]                                                # [B, N]
    end = {"causal": pos + 1, "block": (pre + n)[:, None].expand(B, N), "prefix": pre[:, None].expand(B, N)}[case["mask"]]
    seen = j[None, None] < end[:, :, None]
    if case["window"]:
        seen = seen & ((j[None, None] > (pos - case["window"])[:, :, None]) | (j < case["sinks"])[None, None])
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    o = torch.einsum("bhgns,bshd->bnhgd", e / torch.where(total > 0, total, torch.ones_like(total)), v)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2)             # log 0 = -inf where nothing is seen
    b, at, _ = _places(s)
    return o.reshape(B, N, H, D)[b, at].to(dt), lse.reshape(B, N, H)[b, at].contiguous()


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotate":
        T = case["tokens"]
        return {"bytes": T * (2 * (H + Hk) * D * size + 4), "flops": T * (H + Hk) * D * 7}
    pre, new = _lengths(case)
    if case["op"] == "append":
        T = sum(new)
        return {"bytes": T * (2 * (H + 2 * Hk) * D * size) + case["seqs"] * 12, "flops": T * (H + Hk) * D * 7}
    read, pairs = 0, 0
    w, s0 = case["window"], case["sinks"]
    for p, n in zip(pre, new):
        if n == 0:
            continue
        ends = [p + i + 1 if case["mask"] == "causal" else p + n if case["mask"] == "block" else p for i in range(n)]
        lows = [max(0, p + i + 1 - w) if w else 0 for i in range(n)]
        pairs += sum(max(0, e - lo) + min(s0, lo, e) for e, lo in zip(ends, lows))
        read += max(0, max(ends) - lows[0]) + min(s0, lows[0], max(ends))
    T = sum(new)
    return {"bytes": 2 * read * Hk * D * size + 2 * T * H * D * size + 4 * T * H, "flops": 4 * D * H * pairs}


# ---- the operators' definitions in 64 bits ---------------------------------------------------------------------------

def _turn(x, gamma, at, case):
    """x [T, heads, D] in 64 bits: complex numbers turned by e^(i p w_j)."""
    y = x.double()
    if gamma is not None:
        y = y / (y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + EPS).sqrt() * gamma.double()
    half = case["rot"] // 2
    if half == 0:
        return y
    freq = torch.tensor([THETA ** (-j / half) for j in range(half)], dtype=torch.float64, device=x.device)
    unit = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), at.double().unsqueeze(-1) * freq).unsqueeze(1)
    first = torch.arange(half, device=x.device) * (2 if case["interleaved"] else 1)
    second = first + (1 if case["interleaved"] else half)
    turned = torch.complex(y[..., first], y[..., second]) * unit
    y = y.clone()
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return _turn(s["q"], s.get("gamma_q"), s["positions"], case), _turn(s["k"], s.get("gamma_k"), s["positions"], case)
    pre, new = _lengths(case)
    table, P, D = s["page_table"].tolist(), case["page"], case["dim"]
    if case["op"] == "append":
        at = torch.cat([torch.arange(p, p + n) for p, n in zip(pre, new)]).to(s["q"].device)
        k, q = _turn(s["k"], s.get("gamma_k"), at, case), _turn(s["q"], s.get("gamma_q"), at, case)
        kp, vp, t = s["k_pages"].double(), s["v_pages"].double(), 0
        for b, (p, n) in enumerate(zip(pre, new)):
            done = 0
            while done < n:
                page, row = (p + done) // P, (p + done) % P
                m = min(P - row, n - done)
                kp[table[b][page], :, row:row + m] = k[t + done:t + done + m].transpose(0, 1)
                vp[table[b][page], :, row:row + m] = s["v"][t + done:t + done + m].double().transpose(0, 1)
                done += m
            t += n
        return q, kp, vp
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=s["q"].device)
    group, t = case["heads"] // case["kv_heads"], 0
    for b, (p, n) in enumerate(zip(pre, new)):
        if n == 0:
            continue
        length = p + n
        pages = torch.tensor(table[b][:-(-length // P)], device=s["q"].device)
        key = torch.arange(length, device=s["q"].device)
        at = p + torch.arange(n, device=s["q"].device)[:, None]
        hidden = {"causal": key > at, "block": key >= length, "prefix": key.expand(n, -1) >= p}[case["mask"]]
        if case["window"]:
            hidden = hidden | ((key <= at - case["window"]) & (key >= case["sinks"]))
        for h in range(case["kv_heads"]):
            k = s["k_pages"][pages, h].reshape(-1, D)[:length].double()
            v = s["v_pages"][pages, h].reshape(-1, D)[:length].double()
            for a in range(h * group, (h + 1) * group):
                z = (s["q"][t:t + n, a].double() @ k.T / D ** 0.5).masked_fill(hidden, -math.inf)
                lse[t:t + n, a] = torch.logsumexp(z, -1)
                out[t:t + n, a] = torch.softmax(z, -1).nan_to_num(0.0) @ v
        t += n
    return out, lse

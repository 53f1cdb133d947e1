"""An 8-bit paged key / value cache and the attention of packed rows, operator by operator: cases, inputs, plain forms, work.

What a serving step runs beside the operators of a 16-bit cache:
  append   a step's keys normalised, rotated and quantised, its values quantised, on their way into 8-bit pages (mrp_kv_append_q8)
  read     rows of an 8-bit cache back in the model's type (mrp_kv_read_q8)
  attend   the step's queries over 8-bit pages (mrp_paged_attention_q8)
  packed   prompts over their own keys and values, which lie one sequence after the other and in no cache (mrp_packed_attention)
  block    blocks that are decoded again and again: their queries over the 8-bit cache in front of them, joined with those over the
           block's own keys and values, which are not in the cache yet (mrp_paged_attention_q8, then mrp_packed_attention)

A row (a position's key or value of one head) is held as head_dim e4m3 codes and one scale 2^E, E the smallest integer with
max |row| <= 448 * 2^E (0 for a row of zeros).

`own` false: elementary torch operations in 32 bits (what is quantised: in 64), rounded once at the end.  `own` true: the library's
calls.
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
        # a serving step at the decode shape (d = 2048: 16 heads of 128): 24 sequences, blocks of 4 positions; latency
        dict(name="append blocks", op="append", dtype="bf16", seqs=24, new_lo=4, new_hi=4, pre_lo=50, pre_hi=7000,
             heads=16, kv_heads=8, dim=128, rot=128, interleaved=False, norm=True, page=16, mix=11),
        # ragged prompts of the d = 4096 shape entering the cache
        dict(name="append prompts", op="append", dtype="bf16", seqs=7, new_lo=500, new_hi=3500, pre_lo=0, pre_hi=1500,
             heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, norm=True, page=64, mix=12),
        # 32-bit rows of three short caches, heads of 80, pages of 24
        dict(name="read short f32", op="read", dtype="f32", seqs=3, new_lo=90, new_hi=700, pre_lo=0, pre_hi=40,
             heads=12, kv_heads=4, dim=80, page=24, mix=13),
        # whole caches on their way out (another layout, another model): six sequences
        dict(name="read caches", op="read", dtype="bf16", seqs=6, new_lo=4000, new_hi=20000, pre_lo=0, pre_hi=0,
             heads=32, kv_heads=8, dim=128, page=32, mix=14),
        # one new token of one sequence: latency
        dict(name="attend one token", op="attend", dtype="bf16", seqs=1, new_lo=1, new_hi=1, pre_lo=2500, pre_hi=2500,
             heads=16, kv_heads=8, dim=128, page=16, mask="causal", window=0, sinks=0, mix=15),
        # one token each of 64 ragged sequences
        dict(name="attend 64 ragged", op="attend", dtype="bf16", seqs=64, new_lo=1, new_hi=1, pre_lo=30, pre_hi=9000,
             heads=32, kv_heads=8, dim=128, page=64, mask="causal", window=0, sinks=0, mix=16),
        # a chunk of two prompts behind what is cached already
        dict(name="attend prompt chunk", op="attend", dtype="bf16", seqs=2, new_lo=1800, new_hi=2200, pre_lo=4000, pre_hi=6000,
             heads=32, kv_heads=8, dim=128, page=64, mask="causal", window=0, sinks=0, mix=17),
        # 32-bit queries, odd sizes everywhere, a window and the first tokens
        dict(name="attend odd f32", op="attend", dtype="f32", seqs=7, new_lo=1, new_hi=9, pre_lo=0, pre_hi=3500,
             heads=12, kv_heads=4, dim=72, page=20, mask="causal", window=900, sinks=5, mix=18),
        # blocks of 4 positions that see themselves whole, behind their caches
        dict(name="block of 4", op="block", dtype="bf16", seqs=32, new_lo=4, new_hi=4, pre_lo=200, pre_hi=6000,
             heads=32, kv_heads=8, dim=128, page=32, mask="block", window=0, sinks=0, mix=19),
        # blocks of 32 positions at the decode shape
        dict(name="block of 32", op="block", dtype="bf16", seqs=12, new_lo=32, new_hi=32, pre_lo=500, pre_hi=4500,
             heads=16, kv_heads=8, dim=128, page=128, mask="block", window=0, sinks=0, mix=20),
        # prompts of different lengths, one after the other
        dict(name="packed prompts", op="packed", dtype="bf16", seqs=4, new_lo=600, new_hi=4000, pre_lo=0, pre_hi=0,
             heads=32, kv_heads=8, dim=128, mask="causal", window=0, sinks=0, mix=21),
        # many short prompts, three heads a key head, heads of 80
        dict(name="packed short odd", op="packed", dtype="bf16", seqs=40, new_lo=1, new_hi=70, pre_lo=0, pre_hi=0,
             heads=15, kv_heads=5, dim=80, mask="causal", window=0, sinks=0, mix=22),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "block", "packed"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 4, 5, 8, 16])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 8) if kv * g <= 32])
    dim = rng.choice([64, 128, 128, 128, rng.randrange(4, 33) * 8])
    page = rng.choice([16, 32, 64, 128, rng.randrange(5, 200)])
    seqs = _log(rng, 1, 48)
    mix = rng.randrange(1 << 20)
    base = dict(op=op, dtype=dtype, seqs=seqs, heads=heads, kv_heads=kv, dim=dim, mix=mix)
    if op in ("append", "read"):
        hi = min(_log(rng, 1, 4000), (14000 if dim <= 128 else 7000) // seqs)
        base.update(new_lo=rng.randrange(0, hi + 1), new_hi=hi, pre_lo=0, pre_hi=_log(rng, 1, 1500), page=page)
        if op == "append":
            base.update(rot=rng.choice([dim, dim // 2]), interleaved=rng.random() < 0.3, norm=rng.random() < 0.7)
        return base
    window = rng.choice([0, 0, _log(rng, 1, 4096)])
    if op == "packed":
        new = min(_log(rng, 1, 3500), 9000 // seqs)
        if dtype == "f32" or dim > 128:
            new = min(new, 700)
        return dict(base, new_lo=max(1, new // 4) if rng.random() < 0.6 else new, new_hi=new, pre_lo=0, pre_hi=0,
                    mask=rng.choice(["causal", "causal", "block"]), window=window, sinks=rng.choice([0, 4, 77]) if window else 0)
    long = min(_log(rng, 16, 30000), 100000 // seqs)
    if op == "block":
        new = rng.choice([1, 4, 16, 32, rng.randrange(2, 65)])
        new = max(1, min(new, int(2e7 / (seqs * long))))
        window = 0
    else:
        new = min(_log(rng, 1, 700), 6000 // seqs)
        new = 1 if rng.random() < 0.3 else new if new * seqs * long < 2e7 else max(1, int(2e7 / (seqs * long)))
    if dtype == "f32" or dim > 128:
        long, new = min(long, 30000 // seqs), min(new, 300)
    return dict(base, new_lo=1 if rng.random() < 0.5 else new, new_hi=new, pre_lo=rng.randrange(0, long), pre_hi=long, page=page,
                mask="block" if op == "block" else rng.choice(["causal", "causal", "block", "prefix"]), window=window,
                sinks=rng.choice([0, 4, 77]) if window else 0)


def _lengths(case):
    """(cached tokens, new tokens) of every sequence: part of the case, not of the seed.  Of `read`: (first row, rows)."""
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


def _quantise(x):
    """Rows x [.., D] -> (e4m3 codes, scale bytes E + 127), in the rows' own precision (scaling by a power of two is exact)."""
    top = x.abs().amax(-1)
    part, e = torch.frexp(top)                               # 448 = 0.875 * 2^9
    e = torch.where(top > 0, e - 9 + (part > 0.875), torch.zeros_like(e)).clamp(-127, 127)
    codes = torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    pre, new = _lengths(case)
    B, T, P = case["seqs"], sum(new), case.get("page", 0)
    s = dict(case=case, n_tokens=T, most_new=max(max(new), 1), longest=max(p + n for p, n in zip(pre, new)))
    s["seq_start"] = torch.tensor([0] + list(torch.tensor(new).cumsum(0).tolist()), device=dev, dtype=torch.int32)
    s["prefix_len"] = torch.tensor(pre, device=dev, dtype=torch.int32)
    if P:
        held = [p if case["op"] == "block" else p + n for p, n in zip(pre, new)]
        per = max(1, max(-(-t // P) for t in held))
        used = sum(-(-t // P) for t in held)
        n_pages = used + 3
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        counts = torch.tensor([-(-t // P) for t in held], device=dev)
        col = torch.arange(per, device=dev)
        slot = (counts.cumsum(0) - counts)[:, None] + torch.minimum(col[None], (counts[:, None] - 1).clamp(min=0))
        s["page_table"] = order[slot.clamp(max=n_pages - 1)].contiguous()
        s["longest_cache"] = max(held)
        for x in "kv":                                       # rows of different sizes, as heads and tokens have them
            rows = normal(n_pages, Hk, P, D, dtype=torch.float32) * torch.exp(0.5 * normal(n_pages, Hk, P, 1, dtype=torch.float32))
            s[x + "_codes"], s[x + "_scale"] = _quantise(rows)
            del rows
    s["qkv"] = normal(T, (H + 2 * Hk) * D)
    if case["op"] != "append":
        s["qkv"] *= 1.5                                      # scores spread like those of trained heads
    rows = s["qkv"].view(T, H + 2 * Hk, D)
    s["q"], s["k"], s["v"] = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    if case.get("norm"):
        s["gamma_q"], s["gamma_k"] = 1 + 0.1 * normal(D), 1 + 0.1 * normal(D)
    s["q_out"] = torch.zeros((T, H, D), device=dev, dtype=dt)
    s["lse"] = torch.zeros((T, H), device=dev, dtype=torch.float32)
    if case["op"] == "read":
        s["k_out"], s["v_out"] = (torch.zeros((T, Hk, D), device=dev, dtype=dt) for _ in range(2))
    if own:
        from paper_2605_18817_b200 import binding
        shape = dict(n_heads=H, n_kv_heads=Hk, head_dim=D, page_size=P or 16, rot_dim=case.get("rot", 0),
                     rot_theta=THETA, rot_interleaved=bool(case.get("interleaved")), norm_eps=EPS)
        if P:
            shape.update(n_pages=s["k_codes"].shape[0], max_pages=s["page_table"].shape[1])
        s["ctx"] = _context(dev, case["dtype"], B, shape)
        s["batch"] = binding.KvBatch(s["seq_start"], s["prefix_len"] if P else None, s.get("page_table"), T, s["most_new"])
        if P:
            s["pool"] = binding.KvPoolQ8(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    return {"append": _append, "read": _read, "attend": _attend, "block": _attend, "packed": _attend}[case["op"]](s, case)


def _pools(s):
    """The cache as it stands: codes and scales as the numbers they are."""
    return s["k_codes"], s["v_codes"], s["k_scale"].view(torch.float8_e8m0fnu), s["v_scale"].view(torch.float8_e8m0fnu)


def _run_own(s, case):
    from paper_2605_18817_b200 import binding
    ctx, batch, op = s["ctx"], s["batch"], case["op"]
    if op == "append":
        binding.mrp_kv_append_q8(ctx, batch, s["pool"], s["k"], s["v"], s.get("gamma_k"), s["q"], s["q_out"], s.get("gamma_q"))
        return (s["q_out"],) + _pools(s)
    if op == "read":
        binding.mrp_kv_read_q8(ctx, batch, s["pool"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"]
    how = dict(window=case["window"], sinks=case["sinks"])
    if op == "attend":
        binding.mrp_paged_attention_q8(ctx, batch, s["pool"], s["q"], s["q_out"], s["lse"], mask=MASKS[case["mask"]], **how)
    if op == "block":
        binding.mrp_paged_attention_q8(ctx, batch, s["pool"], s["q"], s["q_out"], s["lse"], mask=PREFIX)
    if op in ("block", "packed"):
        binding.mrp_packed_attention(ctx, batch, s["k"], s["v"], s["q"], s["q_out"], s["lse"], mask=MASKS[case["mask"]],
                                     join=op == "block", **how)
    return s["q_out"], s["lse"]


def _norm_rotate(x, gamma, positions, case):
    """x [T, heads, D] -> the same type: RMSNorm over D, then the first `rot` features turned by their angles."""
    if gamma is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.to(x.dtype)
    rot = case["rot"]
    if rot == 0:
        return x
    j = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
    angle = positions.double()[:, None] * THETA ** (-2.0 * j / rot)
    c, n = angle.cos().to(x.dtype)[:, None], angle.sin().to(x.dtype)[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, w = a * c - b * n, b * c + a * n
    turned = torch.stack((u, w), -1).flatten(-2) if case["interleaved"] else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _places(s):
    """Of every token: its sequence, its place among the sequence's new tokens, its position."""
    t = torch.arange(s["n_tokens"], device=s["seq_start"].device)
    b = torch.searchsorted(s["seq_start"][1:].long(), t, right=True)
    i = t - s["seq_start"].long()[b]
    return b, i, s["prefix_len"].long()[b] + i


def _append(s, case):
    b, _, pos = _places(s)
    page, row = s["page_table"].long()[b, pos // case["page"]], pos % case["page"]
    for x, y in (("k", _norm_rotate(s["k"].double(), s.get("gamma_k"), pos, case)), ("v", s["v"].double())):
        codes, scale = _quantise(y)                          # (next to a border of the codes 32 bits may fall on either side)
        s[x + "_codes"].view(torch.uint8)[page, :, row] = codes.view(torch.uint8)
        s[x + "_scale"][page, :, row] = scale
    return (_norm_rotate(s["q"].float(), s.get("gamma_q"), pos, case).to(s["q"].dtype),) + _pools(s)


def _values(s, x, page, row):
    """Rows of the cache in 32 bits."""
    codes, scale = s[x + "_codes"].view(torch.uint8)[page, :, row].view(torch.float8_e4m3fn), s[x + "_scale"][page, :, row]
    return torch.ldexp(codes.float(), scale.int()[..., None] - 127)


def _read(s, case):
    b, _, pos = _places(s)
    page, row = s["page_table"].long()[b, pos // case["page"]], pos % case["page"]
    return tuple(_values(s, x, page, row).to(s["q"].dtype) for x in "kv")


def _attend(s, case):
    dev, dt, op = s["q"].device, s["q"].dtype, case["op"]
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    B, N, T = case["seqs"], s["most_new"], s["n_tokens"]
    start, pre = s["seq_start"].long(), s["prefix_len"].long()
    n = start[1:] - start[:-1]
    i = torch.arange(N, device=dev)
    own_rows = (start[:-1, None] + i[None]).clamp(max=T - 1)                    # [B, N]
    k, v, at, used = [], [], [], []
    if op != "packed":
        j = torch.arange(s["longest_cache"], device=dev)
        page = s["page_table"].long()[:, j // case["page"]]
        held = pre if op == "block" else pre + n
        k.append(_values(s, "k", page, j % case["page"]))                       # [B, S, Hk, D]
        v.append(_values(s, "v", page, j % case["page"]))
        at.append(j[None].expand(B, -1))
        used.append(j[None] < held[:, None])
    if op != "attend":
        k.append(s["k"][own_rows].float())
        v.append(s["v"][own_rows].float())
        at.append(pre[:, None] + i[None])
        used.append(i[None] < n[:, None])
    at, used = torch.cat(at, 1), torch.cat(used, 1)                             # positions of the keys, which of them there are
    k = torch.cat(k, 1).masked_fill(~used[:, :, None, None], 0.0)
    v = torch.cat(v, 1).masked_fill(~used[:, :, None, None], 0.0)
    q = s["q"][own_rows].float().view(B, N, Hk, H // Hk, D)
    z = torch.einsum("bnhgd,bshd->bhgns", q, k) * (1.0 / math.sqrt(D))
    pos = pre[:, None] + i[None]                                                # [B, N]
    end = {"causal": pos + 1, "block": (pre + n)[:, None].expand(B, N), "prefix": pre[:, None].expand(B, N)}[case["mask"]]
    seen = used[:, None] & (at[:, None] < end[:, :, None])
    if case["window"]:
        seen = seen & ((at[:, None] > (pos - case["window"])[:, :, None]) | (at < case["sinks"])[:, None])
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    o = torch.einsum("bhgns,bshd->bnhgd", e / torch.where(total > 0, total, torch.ones_like(total)), v)
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2)             # log 0 = -inf where nothing is seen
    b, place, _ = _places(s)
    return o.reshape(B, N, H, D)[b, place].to(dt), lse.reshape(B, N, H)[b, place].contiguous()


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    H, Hk, D, op = case["heads"], case["kv_heads"], case["dim"], case["op"]
    pre, new = _lengths(case)
    T, row = sum(new), D + 1                                 # a row of the cache: its codes and its scale
    if op == "append":
        return {"bytes": T * ((2 * H + 2 * Hk) * D * size + 2 * Hk * row) + case["seqs"] * 12, "flops": T * ((H + Hk) * 7 + 2 * Hk * 3) * D}
    if op == "read":
        return {"bytes": T * 2 * Hk * (row + D * size) + case["seqs"] * 12, "flops": T * 2 * Hk * D}
    cached, fresh, pairs = 0, 0, 0
    w, s0 = case["window"], case["sinks"]
    for p, n in zip(pre, new):
        if n == 0:
            continue
        ends = [p + i + 1 if case["mask"] == "causal" else p + n if case["mask"] == "block" else p for i in range(n)]
        lows = [max(0, p + i + 1 - w) if w else 0 for i in range(n)]
        pairs += sum(max(0, e - lo) + min(s0, lo, e) for e, lo in zip(ends, lows))
        read = max(0, max(ends) - lows[0]) + min(s0, lows[0], max(ends))
        own_keys = 0 if op == "attend" else min(n, read)
        fresh += own_keys
        cached += read - own_keys
    return {"bytes": 2 * cached * Hk * row + 2 * fresh * Hk * D * size + 2 * T * H * D * size + 4 * T * H, "flops": 4 * D * H * pairs}


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


def _scale_of(y):
    """2^E of rows, by counting: the powers of two that are too small for the row."""
    powers = 2.0 ** torch.arange(-127, 128, dtype=torch.float64, device=y.device)
    top = y.abs().amax(-1)
    e = torch.searchsorted(448.0 * powers, top.contiguous())   # the first with top <= 448 * 2^E
    return torch.where(top > 0, powers[e.clamp(max=254)], torch.ones_like(top))


def _held(s, x, pages, head):
    """Rows of one key head in pages, in 64 bits: codes taken apart by their bits."""
    c = s[x + "_codes"].view(torch.uint8)[pages, head].long()
    sign, field, part = 1 - 2 * (c >> 7), (c >> 3) & 15, (c & 7).double()
    value = torch.where(field > 0, (1 + part / 8) * 2.0 ** (field - 7).double(), part * 2.0 ** -9)
    value = sign * value * 2.0 ** (s[x + "_scale"][pages, head].double() - 127)[..., None]
    return value.reshape(-1, value.shape[-1])


def exact(case, seed):
    """(The codes of `append` as row / 2^E before their rounding to 8 bits.)"""
    s = prepare(case, seed)
    dev, op = s["q"].device, case["op"]
    pre, new = _lengths(case)
    P, D, Hk = case.get("page", 0), case["dim"], case["kv_heads"]
    table = s["page_table"].tolist() if P else None
    if op == "append":
        at = torch.cat([torch.arange(p, p + n) for p, n in zip(pre, new)]).to(dev)
        rows = dict(k=_turn(s["k"], s.get("gamma_k"), at, case), v=s["v"].double())
        codes, scales = {}, {}
        for x in "kv":
            scale = _scale_of(rows[x])
            codes[x], scales[x], t = s[x + "_codes"].double(), 2.0 ** (s[x + "_scale"].double() - 127), 0
            for b, (p, n) in enumerate(zip(pre, new)):
                done = 0
                while done < n:
                    page, row = (p + done) // P, (p + done) % P
                    m = min(P - row, n - done)
                    part = slice(t + done, t + done + m)
                    codes[x][table[b][page], :, row:row + m] = (rows[x][part] / scale[part][..., None]).transpose(0, 1)
                    scales[x][table[b][page], :, row:row + m] = scale[part].transpose(0, 1)
                    done += m
                t += n
        return _turn(s["q"], s.get("gamma_q"), at, case), codes["k"], codes["v"], scales["k"], scales["v"]
    if op == "read":
        out = []
        for x in "kv":
            got, t = torch.zeros((s["n_tokens"], Hk, D), dtype=torch.float64, device=dev), 0
            for b, (p, n) in enumerate(zip(pre, new)):
                if n > 0:
                    pages = torch.tensor(table[b][:-(-(p + n) // P)], device=dev)
                    for h in range(Hk):
                        got[t:t + n, h] = _held(s, x, pages, h)[p:p + n]
                t += n
            out.append(got)
        return tuple(out)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=dev)
    group, t = case["heads"] // Hk, 0
    for b, (p, n) in enumerate(zip(pre, new)):
        if n == 0:
            continue
        cached = p + n if op == "attend" else p if op == "block" else 0
        key = torch.arange(p + n, device=dev)
        at = p + torch.arange(n, device=dev)[:, None]
        hidden = {"causal": key > at, "block": key >= p + n, "prefix": key.expand(n, -1) >= p}[case["mask"]]
        if case["window"]:
            hidden = hidden | ((key <= at - case["window"]) & (key >= case["sinks"]))
        for h in range(Hk):
            k, v = [], []
            for x, to in (("k", k), ("v", v)):
                if cached > 0:
                    to.append(_held(s, x, torch.tensor(table[b][:-(-cached // P)], device=dev), h)[:cached])
                if op != "attend":
                    to.append(s[x][t:t + n, h].double())
            k, v = torch.cat(k), torch.cat(v)
            for a in range(h * group, (h + 1) * group):
                z = (s["q"][t:t + n, a].double() @ k.T / D ** 0.5).masked_fill(hidden, -math.inf)
                lse[t:t + n, a] = torch.logsumexp(z, -1)
                out[t:t + n, a] = torch.softmax(z, -1).nan_to_num(0.0) @ v
        t += n
    return out, lse

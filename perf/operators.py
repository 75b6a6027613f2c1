"""Operators around the cache whose speed is tracked: the way from a layer's projections to its attention.

  rope     rotary positions of queries or of cached keys (hack_rope)
  qkv      queries and keys normalised per head and rotated, and the projection's q, k and v put into the
           layout of the cache's steps, in one pass (hack_qk_norm_rope)
  append   rows quantised into a cache of 4 bits, and read back (hack_kv4_append, hack_kv4_read)
  attend   attention over a cache of 4 bits: grouped heads, ragged lengths, causal or not, a sliding window
           with first tokens that stay visible (hack_kv4_attend)

With `own` false, `run` computes them from elementary torch operations; with `own` true through the library.

A row of the 4-bit cache: blocks of 16 elements share a scale s, one of the 256 values (1 + m/8) 2^(e-20)
(byte = 8 e + m): the smallest with 7 s >= max |x| of the block, or the largest of all.  An element is
c * s, c = x / s rounded to the nearest whole number (ties to even) within -7..7; byte j of a row holds
c + 8 of element 2j in its low and of element 2j + 1 in its high half.
"""
import math

import torch

own = False

SCALE_BYTES = 256


# ------------------------------------------------------------------ cases
def _rope(name, dtype, batch, heads, tokens, dim, rotary, layout, axes, scaling, far):
    return {"name": name, "op": "rope", "dtype": dtype, "batch": batch, "heads": heads, "tokens": tokens, "dim": dim,
            "rotary": rotary, "layout": layout, "axes": axes, "scaling": scaling, "far": far}


def _qkv(name, dtype, batch, heads, kv_heads, tokens, dim, rotary, layout, axes, norm):
    return {"name": name, "op": "qkv", "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "tokens": tokens,
            "dim": dim, "rotary": rotary, "layout": layout, "axes": axes, "norm": norm}


def _append(name, dtype, batch, kv_heads, tokens, dim, stored):
    return {"name": name, "op": "append", "dtype": dtype, "batch": batch, "kv_heads": kv_heads, "tokens": tokens, "dim": dim,
            "stored": stored}


def _attend(name, dtype, batch, kv_heads, group, tokens, dim, stored, causal=False, sinks=0, window=0):
    return {"name": name, "op": "attend", "dtype": dtype, "batch": batch, "kv_heads": kv_heads, "group": group, "tokens": tokens,
            "dim": dim, "stored": stored, "causal": causal, "sinks": sinks, "window": window}


def listed():
    return [
        # the query of one token: the smallest call there is
        _rope("rope-token", "bf16", 1, 32, 1, 128, 128, "half", 1, "none", 4000),
        # stored keys of 10521 tokens rotated to other positions, half of the head, far positions of a stretched context
        _rope("rope-keys", "f32", 2, 16, 10521, 128, 64, "pairs", 1, "bands", 1000000),
        # the first scale of a stack of 16 heads, conditional and unconditional branch: one token each
        _qkv("qkv-first-scale", "bf16", 2, 16, 16, 1, 128, 128, "half", 2, "l2"),
        # an odd scale of 13 x 13 tokens in fp32
        _qkv("qkv-odd-scale", "f32", 3, 30, 30, 169, 64, 64, "pairs", 2, "rms"),
        # the last scale at 1024 x 1024 of a stack of 32 heads: the largest
        _qkv("qkv-last-scale", "bf16", 2, 32, 32, 4096, 128, 128, "half", 2, "rms"),
        # one token of each of 16 sequences joins their caches
        _append("append-token", "bf16", 16, 16, 1, 64, 2240),
        # the last scale of two images joins
        _append("append-scale", "bf16", 2, 32, 4096, 128, 6425),
        # one token of one sequence over the keys of a whole image
        _attend("attend-token", "bf16", 1, 16, 1, 1, 128, 10521),
        # one token of each of four sequences of up to 65536 keys, four query heads to a stored head
        _attend("attend-long", "bf16", 4, 8, 4, 1, 128, 65536, causal=True),
        # a few queries in fp32, odd everything
        _attend("attend-few-f32", "f32", 3, 5, 3, 13, 64, 2203),
        # a block of a prompt: a window of 1024 and four first tokens
        _attend("attend-window", "bf16", 1, 8, 4, 2240, 64, 10521, causal=True, sinks=4, window=1024),
        # the last scale at 1024 x 1024 over everything stored: the largest
        _attend("attend-last-scale", "bf16", 2, 32, 1, 4096, 128, 10521),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "qkv", "qkv", "append", "attend", "attend", "attend"])
    dim, dtype = rng.choice([64, 128]), rng.choice(["bf16", "bf16", "f32"])
    if op in ("rope", "qkv"):
        axes = rng.choice([1, 2])
        rotary = rng.choice([dim, dim, dim // 2, 2 * axes * rng.randint(1, dim // (2 * axes))])
        layout = rng.choice(["half", "pairs"])
        batch, heads = _log_int(rng, 1, 16), rng.randint(1, 32)
        tokens = _log_int(rng, 1, max(1, min(10521, (2 * 32 * 4096 * 128) // (batch * heads * dim))))
        if op == "rope":
            c = _rope("", dtype, batch, heads, tokens, dim, rotary, layout, axes, rng.choice(["none", "linear", "base", "bands"]),
                      _log_int(rng, 1000, 1000000))
        else:
            group = rng.choice([g for g in (1, 1, 2, 4, 8) if heads % g == 0])
            c = _qkv("", dtype, batch, heads, heads // group, tokens, dim, rotary, layout, axes, rng.choice(["rms", "l2", "none"]))
    elif op == "append":
        batch, heads = _log_int(rng, 1, 16), rng.randint(1, 32)
        tokens = _log_int(rng, 1, max(1, min(4096, (2 * 32 * 4096 * 128) // (batch * heads * dim))))
        c = _append("", dtype, batch, heads, tokens, dim, _log_int(rng, 1, 10521))
    else:
        batch, kv_heads, group = _log_int(rng, 1, 16), _log_int(rng, 1, 32), rng.choice([1, 1, 2, 3, 4, 8])
        tokens, stored = _log_int(rng, 1, 4096), _log_int(rng, 64, 65536)
        causal = rng.random() < 0.5
        windowed = causal and rng.random() < 0.4
        c = _attend("", dtype, batch, kv_heads, group, tokens, dim, stored, causal=causal, sinks=rng.choice([0, 1, 4, 16]) if windowed else 0,
                    window=_log_int(rng, 16, 4096) if windowed else 0)
        # no more logits and operations than the largest listed case has, a sixteenth of them in fp32; no more rows than fit well
        most = 64 * 4096 * 10521 // (16 if dtype == "f32" else 1)
        while c["batch"] * c["kv_heads"] * c["group"] * c["tokens"] * c["stored"] > most:
            big = max(("batch", "kv_heads", "tokens", "stored"), key=lambda k: c[k])
            c[big] = (c[big] + 1) // 2
        while c["batch"] * c["kv_heads"] * c["stored"] > 4 * 1024 * 1024:
            big = max(("batch", "kv_heads", "stored"), key=lambda k: c[k])
            c[big] = (c[big] + 1) // 2
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """Stored rows of every (batch, head): ragged, as caches of heads of different kinds are; the first one is the longest."""
    n = case["batch"] * case["kv_heads"]
    return [case["stored"] - (i * 7919 % 11) * case["stored"] // 24 for i in range(n)]


def _generator(seed):
    return torch.Generator("cuda").manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _frequencies(case, device="cuda"):
    """Radians per position of every rotated pair, and the factor of cosine and sine, for the case's scaling."""
    pairs = case["rotary"] // 2 // case["axes"]
    dim = 2 * pairs                                   # what an axis rotates
    i = torch.arange(pairs, dtype=torch.float64, device=device)
    base, factor, trained = 10000.0, 8.0, 4096.0
    kind = case.get("scaling", "none")
    if kind == "base":
        base = base * factor ** (dim / max(dim - 2, 1))
    f = base ** (-2.0 * i / dim)
    gain = 1.0
    if kind == "linear":
        f = f / factor
    if kind == "bands":
        # pairs that turn more than 32 times within the trained length stay, those that turn less than once are
        # stretched, with a ramp over the pair numbers between
        def pair_of(turns):
            return dim * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(base))
        low, high = max(math.floor(pair_of(32.0)), 0), min(math.ceil(pair_of(1.0)), dim - 1)
        ramp = ((i - low) / max(high - low, 0.001)).clamp(0, 1)
        f = f * (1 - ramp) + f / factor * ramp
        gain = 0.1 * math.log(factor) + 1.0
    return f, gain


def _positions(case, g):
    b, n = case["batch"], case["tokens"]
    if case["axes"] == 2:                             # rows and columns of a token grid, on the scale of the last one
        side = max(1, math.isqrt(n - 1) + 1)
        t = torch.arange(n, device="cuda")
        return torch.stack([t // side, t % side], -1).to(torch.float32) * (64.0 / side) + torch.rand(1, generator=g, device="cuda")
    first = torch.randint(0, case.get("far", 4096), (b, 1), generator=g, device="cuda")
    return (first + torch.arange(n, device="cuda")).to(torch.int32)


def _keys(g, *shape):
    """Rows like stored keys: a few channels of a head are several times larger than the others."""
    x = _normal(g, *shape)
    return x * (1 + 3 * (_normal(g, *shape[:-2], 1, shape[-1]) > 1.5))


def _planes(x, cap):
    """Rows [heads, n, dim] as the bytes of a 4-bit plane of `cap` rows a head, and their values."""
    code, scale_byte, value = _quantise(x)
    heads, n, dim = x.shape
    packed = (code + 8).to(torch.uint8).view(heads, n, dim // 2, 2)
    packed = packed[..., 0] | (packed[..., 1] << 4)
    codes = torch.zeros(heads, cap, dim // 2, dtype=torch.uint8, device=x.device)
    scales = torch.zeros(heads, cap, dim // 16, dtype=torch.uint8, device=x.device)
    codes[:, :n] = packed
    scales[:, :n] = scale_byte.to(torch.uint8)
    return codes.view(-1, dim // 2), scales.view(-1, dim // 16), value


def prepare(case, seed):
    g, dt, op, b, n, dim = _generator(seed), _dtype(case), case["op"], case["batch"], case["tokens"], case["dim"]
    s = {"case": case}
    if op == "rope":
        s["x"] = _normal(g, b, case["heads"], n, dim).to(dt)
        s["y"] = torch.empty_like(s["x"])
        s["positions"] = _positions(case, g)
    if op == "qkv":
        h, kv = case["heads"], case["kv_heads"]
        s["qkv"] = (_normal(g, b, n, h + 2 * kv, dim) * 1.5).to(dt)         # the projection's output
        for name, heads, first in (("q", h, 0), ("k", kv, h), ("v", kv, h + kv)):
            s[name] = s["qkv"][:, :, first:first + heads].transpose(1, 2)
            s[name + "_out"] = torch.empty(b, heads, n, dim, dtype=dt, device="cuda")
        s["q_weight"], s["k_weight"] = 1 + 0.2 * _normal(g, dim), 1 + 0.2 * _normal(g, dim)
        s["q_gain"] = 4 * torch.exp(0.2 * _normal(g, h)) if case["norm"] == "l2" else None
        s["positions"] = _positions(case, g)
    if op in ("append", "attend"):
        kv = case["kv_heads"]
        cap = case["stored"] + (n if op == "append" else 0)
        s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
        if op == "append":
            s["k"] = _keys(g, b, kv, n, dim).to(dt)
            s["v"] = _normal(g, b, kv, n, dim).to(dt)
            s["k_back"], s["v_back"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
            for name in ("k", "v"):
                s[name + "_codes"] = torch.zeros(b * kv * cap, dim // 2, dtype=torch.uint8, device="cuda")
                s[name + "_scales"] = torch.zeros(b * kv * cap, dim // 16, dtype=torch.uint8, device="cuda")
        else:
            s["k_codes"], s["k_scales"], _ = _planes(_keys(g, b * kv, cap, dim).to(torch.bfloat16), cap)
            s["v_codes"], s["v_scales"], _ = _planes(_normal(g, b * kv, cap, dim).to(torch.bfloat16), cap)
            s["q"] = (_normal(g, b, n, kv * case["group"], dim) * 0.7).to(dt).transpose(1, 2)
            s["out"] = torch.empty(b, n, kv * case["group"], dim, dtype=dt, device="cuda").transpose(1, 2)
        s["cap"] = cap
    if own:
        _handles(s)
    return s


def _handles(s):
    """The plan, the handle and the workspace that a program keeps."""
    import paper_2504_09261_b200 as hb
    case = s["case"]
    if case["op"] in ("rope", "qkv"):
        layout = hb.HACK_ROPE_HALF if case["layout"] == "half" else hb.HACK_ROPE_PAIRS
        scaling = {"none": hb.HACK_ROPE_PLAIN, "linear": hb.HACK_ROPE_LINEAR, "base": hb.HACK_ROPE_BASE,
                   "bands": hb.HACK_ROPE_BANDS}[case.get("scaling", "none")]
        s["plan"] = hb.hack_rope_plan(case["dim"], case["rotary"], layout=layout, axes=case["axes"], base=10000.0, scaling=scaling,
                                      factor=8.0, trained_length=4096)
        s["norm"] = {"rms": hb.HACK_NORM_RMS, "l2": hb.HACK_NORM_L2, "none": hb.HACK_NORM_NONE}[case.get("norm", "none")]
    else:
        s["cache"] = hb.HackKv4(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], batch=case["batch"],
                                n_kv_heads=case["kv_heads"], cap=s["cap"])
    if case["op"] == "attend":
        need = s["cache"].hack_kv4_workspace(s["q"], case["stored"], causal=case["causal"], n_sink=case["sinks"], window=case["window"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ one pass
def run(s):
    return {"rope": _run_rope, "qkv": _run_qkv, "append": _run_append, "attend": _run_attend}[s["case"]["op"]](s)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _angles(case, positions):
    """Cosine and sine [batch or 1, 1, tokens, pairs], from angles in 64 bits."""
    f, gain = _frequencies(case)
    p = positions.to(torch.float64)
    a = (p[..., None] * f).flatten(-2)[None] if case["axes"] == 2 else p[..., None] * f
    return (gain * torch.cos(a)).float()[:, None], (gain * torch.sin(a)).float()[:, None]


def _rotate(case, x, cos, sin):
    """The first `rotary` elements of fp32 rows, pair by pair."""
    r = case["rotary"]
    y = x.clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    y[..., first] = x[..., first] * cos - x[..., second] * sin
    y[..., second] = x[..., first] * sin + x[..., second] * cos
    return y


def _run_rope(s):
    case = s["case"]
    if own:
        import paper_2504_09261_b200 as hb
        hb.hack_rope(s["plan"], s["x"], s["y"], s["positions"], stream=_stream())
        return s["y"]
    cos, sin = _angles(case, s["positions"])
    return _rotate(case, s["x"].float(), cos, sin).to(s["x"].dtype)


def _normalise(case, x, weight, gain):
    x = x.float()
    if case["norm"] == "none":
        return x
    if case["norm"] == "rms":
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    else:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True)).clamp_min(1e-6)
    x = x * weight
    return x if gain is None else x * gain[:, None, None]


def _run_qkv(s):
    case = s["case"]
    if own:
        import paper_2504_09261_b200 as hb
        weights = {} if case["norm"] == "none" else dict(q_weight=s["q_weight"], k_weight=s["k_weight"], q_gain=s["q_gain"])
        hb.hack_qk_norm_rope(s["plan"], s["q"], s["k"], s["v"], s["q_out"], s["k_out"], s["v_out"], s["positions"], norm=s["norm"],
                             eps=1e-6, stream=_stream(), **weights)
        return s["q_out"], s["k_out"], s["v_out"]
    cos, sin = _angles(case, s["positions"])
    q = _rotate(case, _normalise(case, s["q"], s["q_weight"], s["q_gain"]), cos, sin)
    k = _rotate(case, _normalise(case, s["k"], s["k_weight"], None), cos, sin)
    return q.to(s["q"].dtype), k.to(s["k"].dtype), s["v"].contiguous()


def _scale_values(device):
    byte = torch.arange(SCALE_BYTES, device=device)
    return (1 + (byte % 8).float() / 8) * torch.exp2((byte // 8).float() - 20)


def _quantise(x):
    """Codes, scale bytes and values (fp32) of rows [..., dim].  Divided in 64 bits: what lies next to the middle
    between two codes would round to the other side in 32."""
    blocks = torch.nan_to_num(x.double(), nan=0.0).unflatten(-1, (-1, 16))
    table = _scale_values(x.device)
    byte = torch.searchsorted(7 * table.double(), blocks.abs().amax(-1)).clamp_max(SCALE_BYTES - 1)
    scale = table[byte][..., None]
    code = torch.round(blocks / scale.double()).clamp(-7, 7)
    value = code.float() * scale
    return code.to(torch.int8).flatten(-2), byte, value.flatten(-2)


def _run_append(s):
    if own:
        cache, stream = s["cache"], _stream()
        cache.hack_kv4_append(s["k"], s["v"], s["lens"], stream=stream)
        cache.hack_kv4_read(s["k_back"], s["v_back"], s["lens"], stream=stream)
        return s["k_back"], s["v_back"]
    return _quantise(s["k"])[2].to(s["k"].dtype), _quantise(s["v"])[2].to(s["v"].dtype)


def _values(s, which):
    """Stored rows [batch, kv_heads, cap, dim] as the values they stand for."""
    case, codes = s["case"], s[which + "_codes"]
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(torch.int8) - 8
    scale = _scale_values(codes.device)[s[which + "_scales"].long()]
    return (c.float().unflatten(-1, (-1, 16)) * scale[..., None]).view(case["batch"], case["kv_heads"], s["cap"], case["dim"])


def _visible(case, lens, cap):
    """[batch, kv_heads, 1, tokens, cap]: which stored rows a query sees.  Query i of n is at position length - n + i."""
    n = case["tokens"]
    length = lens.view(case["batch"], case["kv_heads"], 1, 1, 1).long()
    j = torch.arange(cap, device=lens.device)
    at = length - n + torch.arange(n, device=lens.device)[:, None]
    see = (j < length).expand(-1, -1, -1, n, -1)
    if case["causal"]:
        see = see & (j <= at)
    if case["window"]:
        see = see & ((j < case["sinks"]) | (j > at - case["window"]))
    return see


def _run_attend(s):
    case = s["case"]
    if own:
        s["cache"].hack_kv4_attend(s["q"], s["out"], s["lens"], case["stored"], workspace=s["workspace"], causal=case["causal"],
                                   n_sink=case["sinks"], window=case["window"], stream=_stream())
        return s["out"]
    k, v = _values(s, "k")[:, :, None], _values(s, "v")[:, :, None]
    q = s["q"].float().unflatten(1, (case["kv_heads"], case["group"]))
    logits = torch.matmul(q * case["dim"] ** -0.5, k.transpose(-1, -2))
    logits = logits.masked_fill(~_visible(case, s["lens"], s["cap"]), -math.inf)
    top = logits.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = torch.exp(logits - top)
    out = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).tiny)
    return out.flatten(1, 2).to(s["q"].dtype)


# ------------------------------------------------------------------ what a pass cannot do without
def _pairs(case):
    """Visible (query, key) pairs of one query head of each stored head, summed over the stored heads, and the rows seen."""
    n, pairs, rows = case["tokens"], 0, 0
    for length in _lengths(case):
        at = torch.arange(length - n, length, dtype=torch.int64)
        hi = (at + 1).clamp(0, length) if case["causal"] else torch.full((n,), length)
        lo = (at - case["window"] + 1).clamp_min(0) if case["window"] else torch.zeros(n, dtype=torch.int64)
        sinks = torch.full((n,), case["sinks"] if case["window"] else 0)
        lo = torch.minimum(lo, hi)
        first = torch.minimum(torch.minimum(sinks, lo), hi)        # sinks that lie ahead of the window
        pairs += int((hi - lo + first).sum())
        rows += int(hi.max() - lo.min()) + int(min(int(first.max()), int(lo.min())))
    return pairs, rows


def work(case):
    op, dim, n, size = case["op"], case["dim"], case["tokens"], 4 if case["dtype"] == "f32" else 2
    row4 = dim // 2 + dim // 16
    if op == "rope":
        x = case["batch"] * case["heads"] * n * dim
        positions = 4 * n * (2 if case["axes"] == 2 else case["batch"])
        return {"bytes": 2 * size * x + positions, "flops": 3 * x * case["rotary"] // dim}
    if op == "qkv":
        rows = case["batch"] * n
        x = rows * (case["heads"] + 2 * case["kv_heads"]) * dim
        positions = 4 * n * (2 if case["axes"] == 2 else case["batch"])
        return {"bytes": 2 * size * x + positions, "flops": 8 * rows * (case["heads"] + case["kv_heads"]) * dim}
    if op == "append":
        rows = 2 * case["batch"] * case["kv_heads"] * n
        # read, stored, fetched back and written out
        return {"bytes": rows * (2 * size * dim + 2 * row4), "flops": 4 * rows * dim}
    pairs, rows = _pairs(case)
    q = case["batch"] * case["kv_heads"] * case["group"] * n * dim
    return {"bytes": 2 * size * q + 2 * rows * row4, "flops": 4 * pairs * case["group"] * dim}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_rotation(case, x, positions):
    """x: [b, h, n, d] in 64 bits.  Every pair as a complex number times exp(i angle)."""
    f, gain = _frequencies(case)
    r, p = case["rotary"], positions.to(torch.float64)
    if case["axes"] == 1:
        angle = p[:, None, :, None] * f
    else:
        angle = torch.cat([p[:, 0, None] * f, p[:, 1, None] * f], -1)[None, None]
    rot, rest = x[..., :r], x[..., r:]
    z = torch.complex(rot[..., :r // 2], rot[..., r // 2:]) if case["layout"] == "half" else torch.complex(rot[..., 0::2], rot[..., 1::2])
    z = z * torch.polar(torch.full_like(angle, gain), angle)
    rot = torch.cat([z.real, z.imag], -1) if case["layout"] == "half" else torch.view_as_real(z).flatten(-2)
    return torch.cat([rot, rest], -1)


def _exact_blocks(x):
    """Rows [..., dim] as a 4-bit cache holds them, scale by scale from the definition."""
    blocks = x.double().reshape(-1, 16)
    top = blocks.abs().max(-1).values
    scale = torch.full_like(top, 1.875 * 2.0 ** 11)
    for byte in range(SCALE_BYTES - 1, -1, -1):
        s = (8 + byte % 8) / 8 * 2.0 ** (byte // 8 - 20)
        scale = torch.where(7 * s >= top, torch.full_like(top, s), scale)
    return ((blocks / scale[:, None]).round().clamp(-7, 7) * scale[:, None]).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        return _exact_rotation(case, s["x"].double(), s["positions"])
    if op == "qkv":
        out = []
        for name in ("q", "k"):
            x = s[name].double()
            if case["norm"] != "none":
                weight = s[name + "_weight"].double()
                if name == "q" and s["q_gain"] is not None:
                    weight = weight * s["q_gain"].double().view(-1, 1, 1)
                size = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
                x = weight * x / ((size ** 2 / case["dim"] + 1e-6).sqrt() if case["norm"] == "rms" else size.clamp_min(1e-6))
            out.append(_exact_rotation(case, x, s["positions"]))
        return out[0], out[1], s["v"].double()
    if op == "append":
        return _exact_blocks(s["k"]), _exact_blocks(s["v"])
    n, dim, group, lens = case["tokens"], case["dim"], case["group"], _lengths(case)
    unit = torch.tensor([(8 + i % 8) / 8 * 2.0 ** (i // 8 - 20) for i in range(SCALE_BYTES)], dtype=torch.float64, device="cuda")
    out = torch.zeros(case["batch"], case["kv_heads"] * group, n, dim, dtype=torch.float64, device="cuda")
    for i, length in enumerate(lens):
        b, h = divmod(i, case["kv_heads"])
        at = slice(i * s["cap"], i * s["cap"] + length)
        k, v = (torch.stack([s[w + "_codes"][at] % 16, s[w + "_codes"][at] // 16], -1).reshape(length, dim).double().sub(8)
                * unit[s[w + "_scales"][at].long()].repeat_interleave(16, -1) for w in ("k", "v"))
        j = torch.arange(length, device="cuda")[None]
        p = torch.arange(length - n, length, device="cuda")[:, None]
        hidden = torch.zeros(n, length, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= j > p
        if case["window"]:
            hidden |= (j <= p - case["window"]) & (j >= case["sinks"])
        empty = hidden.all(-1)
        for g in range(group):
            z = s["q"][b, h * group + g].double() @ k.T / math.sqrt(dim)
            o = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ v
            out[b, h * group + g] = torch.where(empty[:, None], torch.zeros_like(o), o)
    return out

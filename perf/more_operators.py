"""The cases on which the rotary and 8-bit paged cache operators are measured, with their plain forms.

Three operators that belong to one step of a server whose keys and values lie in 8-bit pages:

  rope    rotary positions of queries or keys (``mkv_rope_apply``): both layouts, part of a head, tables scaled for long
          contexts, and the transpose that carries gradients back
  append  a step's or a prompt's tokens join the cache (``mkv_paged_append``): queries and keys rotated, keys and values
          quantized to 8 bits (e4m3 or int8) with one power-of-two scale for each page and key head
  attend  causal attention of every entry's newest tokens over its pages (``mkv_paged_attention``): one token an entry,
          a few drafted ones, the next chunk of a prompt or a whole one

``own = False`` computes them with elementary torch operations in 32 bits; ``own = True`` calls the library.
"""
import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}            # the largest code
E_MIN, E_MAX = -100, 120                        # exponents that a page's scale may take


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one decode step of a batch of eight: its query and key heads in one call; latency counts
        dict(name="rope_token", op="rope", dtype="fp16", n=8, heads=40, D=128, rot=128, layout="half", scaling="plain",
             first=8192, wide=40, grad=False),
        # an 8K prompt behind a long context, frequencies scaled in bands
        dict(name="rope_prompt", op="rope", dtype="bf16", n=8192, heads=40, D=128, rot=128, layout="half",
             scaling="bands", first=100000, wide=40, grad=False),
        # the gradient of interleaved, half-rotated heads lying within wider rows, an odd number of tokens
        dict(name="rope_part_grad", op="rope", dtype="bf16", n=1001, heads=12, D=64, rot=32, layout="pairs",
             scaling="ramp", first=4000, wide=17, grad=True),
        # the new token of the library's own decode benchmark's batch and context
        dict(name="append_token", op="append", dtype="fp16", fmt="e4m3", B=8, Hq=32, Hkv=8, D=128, page=16, n=1, T=8192,
             ragged=False, layout="half"),
        # up to nine accepted tokens of each of 64 conversations of unequal lengths
        dict(name="append_accepted", op="append", dtype="bf16", fmt="int8", B=64, Hq=32, Hkv=8, D=128, page=32, n=9,
             T=3001, ragged=True, layout="half"),
        # three prompts of unequal lengths, the first of them behind a cached beginning
        dict(name="append_prompts", op="append", dtype="bf16", fmt="e4m3", B=3, Hq=32, Hkv=8, D=128, page=64, n=4096,
             T=1500, ragged=True, layout="pairs"),
        # a chat's first replies: one token of one conversation, an odd length; latency counts
        dict(name="attend_token_short", op="attend", dtype="bf16", fmt="int8", B=1, Hq=32, Hkv=8, D=128, page=16, n=1,
             T=777, ragged=False),
        # the batch and context of the library's own decode benchmark, one token an entry
        dict(name="attend_token_batch", op="attend", dtype="fp16", fmt="e4m3", B=8, Hq=32, Hkv=8, D=128, page=16, n=1,
             T=8192, ragged=False),
        # long conversations of unequal lengths
        dict(name="attend_token_long", op="attend", dtype="bf16", fmt="int8", B=16, Hq=32, Hkv=8, D=128, page=64, n=1,
             T=32768, ragged=True),
        # up to eight drafted tokens an entry
        dict(name="attend_drafted", op="attend", dtype="fp16", fmt="e4m3", B=8, Hq=32, Hkv=8, D=128, page=32, n=8,
             T=8192, ragged=True),
        # the next chunks of two prompts behind what they have in the cache
        dict(name="attend_chunks", op="attend", dtype="bf16", fmt="int8", B=2, Hq=32, Hkv=8, D=128, page=64, n=511,
             T=8192, ragged=True),
        # a whole prompt
        dict(name="attend_prompt", op="attend", dtype="fp16", fmt="e4m3", B=1, Hq=32, Hkv=8, D=128, page=64, n=4096,
             T=4096, ragged=False),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "append", "attend", "attend", "attend"])
    dtype = rng.choice(["fp16", "bf16"])
    if op == "rope":
        D = rng.choice([64, 80, 128, 192, 256])
        heads = _log(rng, 1, 40)
        n = _log(rng, 1, 8192 * 40 * 128 // (heads * D))
        return dict(op="rope", dtype=dtype, n=min(n, 30000), heads=heads, D=D,
                    rot=rng.choice([D, D, D // 2, 8 * rng.randint(1, D // 8)]), layout=rng.choice(["half", "pairs"]),
                    scaling=rng.choice(["plain", "linear", "bands", "ramp"]), first=rng.randint(0, 100000),
                    wide=heads + rng.choice([0, 0, rng.randint(0, 8)]), grad=rng.random() < 0.3)
    fmt, D, page = rng.choice(["e4m3", "int8"]), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 4, 7, 8])
    B = _log(rng, 1, 64)
    ragged = rng.random() < 0.6
    if op == "append":
        n = _log(rng, 1, 4096)
        while B * n > 3 * 4096:
            n = max(1, n // 2)
        return dict(op="append", dtype=dtype, fmt=fmt, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, n=n,
                    T=_log(rng, 1, 8192), ragged=ragged, layout=rng.choice(["half", "pairs"]))
    kind = rng.choice(["token", "token", "drafted", "chunk"])
    n = {"token": 1, "drafted": _log(rng, 2, 32), "chunk": _log(rng, 33, 4096)}[kind]
    T = n + (0 if kind == "chunk" and rng.random() < 0.3 else _log(rng, 1, 32768 - n))
    while B > 1 and (B * T > 12 * 32768 or B * n * Hkv * G * T > 32 * 4096 * 4096 // 2):
        B //= 2
    while n * Hkv * G * T > 32 * 4096 * 4096 // 2:
        n, T = max(1, n // 2), max(1, T // 2)
    return dict(op="attend", dtype=dtype, fmt=fmt, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, page=page, n=n, T=max(T, n),
                ragged=ragged)


def _lengths(c):
    """Cached tokens of each entry (append: before the call; attend: the new ones among them): all T, or (ragged) unequal
    ones from T down to about T / 2."""
    B, T = c["B"], c["T"]
    return [T - (b * T) // (2 * B) for b in range(B)] if c["ragged"] else [T] * B


def _new(c):
    """New tokens of each entry: n, or (ragged) unequal ones from n down; an attending entry holds them already."""
    B, n = c["B"], c["n"]
    new = [max(1, n - (b * n) // (2 * B) - b % 3) for b in range(B)] if c["ragged"] else [n] * B
    return [min(m, t) for m, t in zip(new, _lengths(c))] if c["op"] == "attend" else new


def work(c):
    """What one pass cannot do without: each input read once, each output written once, each visible pair."""
    if c["op"] == "rope":
        return {"bytes": 4 * c["n"] * c["heads"] * c["D"] + c["n"] * (4 * c["rot"] + 4),
                "flops": 3 * c["n"] * c["heads"] * c["rot"]}
    D, Hq, Hkv, new, lens = c["D"], c["Hq"], c["Hkv"], _new(c), _lengths(c)
    n = sum(new)
    if c["op"] == "append":
        pages = sum((t + m - 1) // c["page"] - t // c["page"] + 1 for t, m in zip(lens, new))
        return {"bytes": n * D * (4 * Hq + 4 * Hkv + 2 * Hkv + 4) + pages * (8 * Hkv + 4) + 8 * c["B"],
                "flops": n * D * (3 * Hq + 7 * Hkv)}
    pages = sum(-(-t // c["page"]) for t in lens)
    pairs = sum(m * (t - m) + m * (m + 1) / 2 for t, m in zip(lens, new))
    return {"bytes": 2 * sum(lens) * Hkv * D + pages * (8 * Hkv + 4) + 4 * n * Hq * D, "flops": 4 * D * Hq * pairs}


# ------------------------------------------------------------------------------------------------ the inputs
def _frequencies(c, dev):
    """Radians a position of each rotated pair, in 64 bits."""
    r, theta = c.get("rot", c["D"]), 500000.0 if c.get("scaling") == "bands" else 10000.0
    i = torch.arange(r // 2, dtype=torch.float64, device=dev)
    f = torch.pow(torch.tensor(theta, dtype=torch.float64, device=dev), -2.0 * i / r)
    kind = c.get("scaling", "plain")
    if kind == "linear":
        return f / 4.0
    if kind == "bands":       # wavelengths up to context / 4 as they are, from context / 1 on divided, between them mixed
        turns = 8192.0 * f / (2.0 * math.pi)
        mix = ((turns - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return (1.0 - mix) * f / 8.0 + mix * f
    if kind == "ramp":        # pairs that turn 32 times within the context as they are, up to those that turn once
        at = [r * math.log(4096.0 / (beta * 2.0 * math.pi)) / (2.0 * math.log(theta)) for beta in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        mix = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return (1.0 - mix) * f / 16.0 + mix * f
    return f


def _table(c, rows, dev):
    """(cos, sin) of each position's angles, worked out in 64 bits: what a program keeps for all of its layers."""
    a = torch.arange(rows, dtype=torch.float64, device=dev)[:, None] * _frequencies(c, dev)
    size = 0.1 * math.log(16.0) + 1.0 if c.get("scaling") == "ramp" else 1.0
    return torch.stack([torch.cos(a) * size, torch.sin(a) * size], -1).float()


def prepare(c, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[c["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).mul_(std).to(dt)

    s = dict(c)
    if c["op"] == "rope":
        n, rows = c["n"], c["first"] + c["n"] + 64
        s["x"] = normal(n, c["wide"], c["D"])[:, :c["heads"]]
        s["pos"] = (c["first"] + torch.arange(n, device=dev) + torch.randint(0, 64, (n,), generator=gen, device=dev)).int()
        s["out"] = torch.empty(n, c["heads"], c["D"], dtype=dt, device=dev)
        s["plan"] = _plan(c, s, rows) if own else {"table": _table(c, rows, dev)}
        return s
    B, Hkv, D, page = c["B"], c["Hkv"], c["D"], c["page"]
    lens, new = _lengths(c), _new(c)
    n = sum(new)
    most = -(-(max(lens) + c["n"]) // page)              # pages an entry may hold
    num = B * most + 3
    s["n_all"], s["num_pages"], s["max_pages"] = n, num, most
    s["page_table"] = torch.randperm(num, generator=gen, device=dev)[:B * most].reshape(B, most).int()
    # codes as quantized standard normals have them, scales that differ from page to page and head to head
    for name in ("k", "v"):
        x = torch.randn((num, Hkv, page, D), generator=gen, device=dev, dtype=torch.float32)
        if c["fmt"] == "int8":
            s[name] = x.mul_(32.0).round_().clamp_(-127, 127).to(torch.int8)
        else:
            s[name] = x.mul_(112.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
        del x
    e = torch.randint(-1, 2, (2, num, Hkv), generator=gen, device=dev)
    base = 2.0 ** -5 if c["fmt"] == "int8" else 2.0 ** -7
    if c["op"] == "append":
        s["k_scale"], s["v_scale"] = (torch.ldexp(torch.full((num, Hkv), base, device=dev), e[j]) for j in (0, 1))
        # keys and values of a token in a wider row, as a fused projection leaves them
        qkv = normal(n, c["Hq"] + 2 * Hkv, D)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :c["Hq"]], qkv[:, c["Hq"]:c["Hq"] + Hkv], qkv[:, c["Hq"] + Hkv:]
        s["q_out"] = torch.empty(n, c["Hq"], D, dtype=dt, device=dev)
        s["T_before"] = torch.tensor(lens, dtype=torch.int32, device=dev)
        s["T_len"] = s["T_before"].clone()
    else:
        # (as another program's calibration may have left them: no powers of two)
        r = torch.rand((2, num, Hkv), generator=gen, device=dev) * 0.5 + 0.75
        s["k_scale"], s["v_scale"] = (torch.ldexp(base * r[j], e[j]) for j in (0, 1))
        s["q"] = normal(n, c["Hq"], D)
        s["out"] = torch.empty(n, c["Hq"], D, dtype=dt, device=dev)
        s["T_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    s["start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
    rows = max(lens) + c["n"]
    s["plan"] = _plan(c, s, rows) if own else {"table": _table(c, rows, dev) if c["op"] == "append" else None}
    return s


def _plan(c, s, rows):
    """What a program that uses the library keeps beside its tensors: configurations, tables, the cache's struct, a
    workspace."""
    import paper_2609_07966_gb300 as mkv
    from paper_2609_07966_gb300 import caches
    p = {"mkv": mkv, "dtype": mkv.MKV_BF16 if c["dtype"] == "bf16" else mkv.MKV_F16}
    if c["op"] != "attend":
        kw = {"plain": {}, "linear": dict(scaling=mkv.MKV_ROPE_LINEAR, factor=4.0),
              "bands": dict(scaling=mkv.MKV_ROPE_BANDS, theta=500000.0, factor=8.0, low=1.0, high=4.0, context=8192),
              "ramp": dict(scaling=mkv.MKV_ROPE_RAMP, factor=16.0, low=1.0, high=32.0, context=4096)}
        p["rope"] = mkv.rope_config(c["D"], rot_dim=c.get("rot", c["D"]),
                                    layout=mkv.MKV_ROPE_PAIRS if c["layout"] == "pairs" else mkv.MKV_ROPE_HALF,
                                    **kw[c.get("scaling", "plain")])
        p["table"] = caches.rope_table(p["rope"], rows)
        p["rows"] = rows
    if c["op"] != "rope":
        p["cfg"] = mkv.paged_config(p["dtype"], mkv.MKV_E4M3 if c["fmt"] == "e4m3" else mkv.MKV_I8, c["B"], c["Hq"],
                                    c["Hkv"], c["D"], c["page"])
        p["cache"] = caches.wrap_paged_cache(p["cfg"], s["page_table"], s["T_len"], s["k"], s["v"], s["k_scale"],
                                             s["v_scale"])
        p["start"] = s["start"].data_ptr() if c["ragged"] else 0
        if c["op"] == "attend":
            p["ws"], p["ws_bytes"] = caches.paged_workspace(p["cfg"], s["n_all"], c["n"])
    return p


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _own(s)
    return {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend}[s["op"]](s)


def _codes(s):
    """The cache's state, its codes as the numbers that they are."""
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "T_len": s["T_len"]}


def _own(s):
    p = s["plan"]
    mkv = p["mkv"]
    if s["op"] == "rope":
        mkv.mkv_rope_apply(p["rope"], p["dtype"], s["x"].data_ptr(), s["wide"] * s["D"], s["pos"].data_ptr(), s["n"],
                           s["heads"], p["table"].data_ptr(), p["rows"], s["grad"], s["out"].data_ptr(), 0)
        return {"out": s["out"]}
    if s["op"] == "append":
        s["T_len"].copy_(s["T_before"])       # the lengths before the step, so that a pass can be repeated
        row = (s["Hq"] + 2 * s["Hkv"]) * s["D"]
        new = mkv.paged_rows(s["n_all"], start=p["start"], q=s["q"].data_ptr(), q_stride=row, k=s["k_new"].data_ptr(),
                             k_stride=row, v=s["v_new"].data_ptr(), v_stride=row, q_out=s["q_out"].data_ptr())
        mkv.mkv_paged_append(p["cfg"], p["rope"], p["table"].data_ptr(), p["rows"], new, p["cache"].c)
        return {"q": s["q_out"], **_codes(s)}
    mkv.mkv_paged_attention(p["cfg"], s["q"].data_ptr(), 0, p["start"], s["n_all"], s["n"], p["cache"].c,
                            s["out"].data_ptr(), 0, p["ws"].data_ptr(), p["ws_bytes"])
    return {"out": s["out"]}


def _rotate(x, cs, layout):
    """The first dims of x [n][heads][D] rotated by (cos, sin) [n][r / 2][2], in 32 bits."""
    r = 2 * cs.shape[1]
    c, t = cs[:, None, :, 0], cs[:, None, :, 1]
    x = x.float()
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * t, b * c + a * t], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * t, b * c + a * t], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_rope(s):
    cs = s["plan"]["table"][s["pos"].long()]
    if s["grad"]:
        cs = cs * torch.tensor([1.0, -1.0], device=cs.device)
    return {"out": _rotate(s["x"], cs, s["layout"]).to(s["x"].dtype)}


def _tokens(s):
    """Entry and place within it of each of the flattened tokens."""
    at = torch.arange(s["n_all"], device=s["start"].device)
    b = torch.searchsorted(s["start"][1:].long(), at, right=True)
    return b, at - s["start"].long()[b]


def _exponent(most, fmt):
    """The least e with most <= top 2^e."""
    m, e = torch.frexp(most)
    over = m > (0.875 if fmt == "e4m3" else 127.0 / 128.0)
    e = e - (9 if fmt == "e4m3" else 7) + over.int()
    return torch.where(most > 0, e, torch.full_like(e, E_MIN)).clamp(E_MIN, E_MAX)


def _encode(x, fmt):
    if fmt == "int8":
        return x.round().clamp(-127.0, 127.0).to(torch.int8)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _plain_append(s):
    fmt, page, Hkv = s["fmt"], s["page"], s["Hkv"]
    b, i = _tokens(s)
    before = s["T_before"].long()
    pos = before[b] + i
    cs = s["plan"]["table"][pos]
    q = _rotate(s["q"], cs, s["layout"]).to(s["q"].dtype)
    pid = s["page_table"].long()[b, pos // page]
    # the page that each entry writes into first, with the tokens that it holds already
    first = s["page_table"].long()[torch.arange(s["B"], device=b.device), (before // page).clamp(max=s["max_pages"] - 1)]
    held = torch.where(s["start"][1:] > s["start"][:-1], before % page, 0)
    fresh = torch.zeros(s["num_pages"], dtype=torch.bool, device=b.device).index_fill_(0, pid, True)
    touched = fresh.clone()
    fresh[first] = fresh[first] & (held == 0)
    for name, x in (("k", _rotate(s["k_new"], cs, s["layout"])), ("v", s["v_new"].float())):
        scale, raw = s[name + "_scale"], s[name].view(torch.uint8 if fmt == "e4m3" else torch.int8)
        most = torch.zeros(s["num_pages"], Hkv, device=b.device)
        most.scatter_reduce_(0, pid[:, None].expand(-1, Hkv), x.abs().amax(-1), "amax")
        was = torch.frexp(scale)[1] - 1
        e = _exponent(most, fmt)
        e = torch.where(fresh[:, None], e, torch.maximum(e, was))
        e = torch.where(touched[:, None], e, was)
        old = raw[first]
        less = torch.ldexp(torch.ones_like(scale[first]), (was - e)[first])[:, :, None, None]
        again = _encode(s[name][first].float() * less, fmt)
        keep = torch.arange(page, device=b.device)[None, None, :, None] < held[:, None, None, None]
        raw[first] = torch.where(keep, again, old)
        raw[pid, :, pos % page] = _encode(torch.ldexp(x, -e[pid][..., None]), fmt)
        scale.copy_(torch.where(touched[:, None], torch.ldexp(torch.ones_like(scale), e), scale))
    s["T_len"].copy_(before + (s["start"][1:] - s["start"][:-1]))
    return {"q": q, **_codes(s)}


def _plain_attend(s):
    B, n, Hq, Hkv, D, page = s["B"], s["n"], s["Hq"], s["Hkv"], s["D"], s["page"]
    G, T = Hq // Hkv, s["max_pages"] * page
    table = s["page_table"].long()

    def values(codes, scale):            # [B][Hkv][T][D]
        x = codes[table].float() * scale[table][..., None, None]
        return x.transpose(1, 2).reshape(B, Hkv, T, D)

    b, i = _tokens(s)
    q = torch.zeros(B, n, Hq, D, device=b.device)
    q[b, i] = s["q"].float()
    q = q.reshape(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    sc = (q @ values(s["k"], s["k_scale"]).transpose(2, 3)) * (1.0 / math.sqrt(D))
    new = s["start"][1:] - s["start"][:-1]
    at = (s["T_len"] - new)[:, None] + torch.arange(n, device=b.device)       # each query's own place
    vis = torch.arange(T, device=b.device) <= at.repeat_interleave(G, 1)[..., None]
    sc = torch.where(vis[:, None], sc, torch.full_like(sc, -3.0e38))
    e = torch.exp(sc - sc.amax(-1, keepdim=True))
    o = (e @ values(s["v"], s["v_scale"])) / e.sum(-1, keepdim=True)
    o = o.reshape(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    return {"out": o[b, i].to(s["q"].dtype)}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(c, seed):
    """The definitions in 64 bits, token by token or entry by entry.  Rotations take angles that were never rounded; an
    append's codes are those of its 32-bit arithmetic, so only its queries have a value here."""
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["op"] == "attend":
        return {"out": _exact_attend(c, s)}
    if c["op"] == "rope":
        return {"out": _exact_rotate(s["x"], s["pos"], c, -1.0 if c["grad"] else 1.0)}
    pos = torch.cat([t + torch.arange(m, device="cuda") for t, m in zip(_lengths(c), _new(c))])
    return {"q": _exact_rotate(s["q"], pos, c, 1.0), "k": None, "v": None, "k_scale": None, "v_scale": None, "T_len": None}


def _exact_rotate(x, pos, c, sign):
    """Pairs as complex numbers, turned by multiplication."""
    x = x.double()
    out, r = x.clone(), c.get("rot", c["D"])
    lo, hi = (slice(0, r // 2), slice(r // 2, r)) if c["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    size = 0.1 * math.log(16.0) + 1.0 if c.get("scaling") == "ramp" else 1.0
    angle = sign * pos.double()[:, None, None] * _frequencies(c, x.device)
    z = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.full_like(angle, size), angle)
    out[..., lo], out[..., hi] = z.real, z.imag
    return out


def _exact_attend(c, s):
    D, G, page = c["D"], c["Hq"] // c["Hkv"], c["page"]
    out, row = [], 0
    for b, (t, m) in enumerate(zip(_lengths(c), _new(c))):
        ids = s["page_table"][b, :-(-t // page)].long()
        k, v = ((s[x][ids].double() * s[x + "_scale"][ids].double()[:, :, None, None]).transpose(0, 1).flatten(1, 2)[:, :t]
                for x in ("k", "v"))
        heads = []
        for h in range(c["Hq"]):
            z = s["q"][row:row + m, h].double() @ k[h // G].T / math.sqrt(D)
            z = z.masked_fill(torch.ones(m, t, dtype=torch.bool, device="cuda").triu(t - m + 1), -math.inf)
            heads.append(torch.softmax(z, -1) @ v[h // G])
        out.append(torch.stack(heads, 1))
        row += m
    return torch.cat(out)

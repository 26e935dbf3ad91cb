"""The cases on which the tree and latent operators are measured, with their plain forms.

Five operators that belong to one serving loop with drafted tokens:

  latent    attention of queries already carried into the latent space over a cache of one shared latent row a
            token (``mkv_latent_attention``): a single token per entry, or a tree of drafted tokens
  product   the per-head products around it (``mkv_latent_absorb``, ``mkv_latent_project``, ``mkv_latent_expand``)
  prefill   the expanded form: causal attention of a prompt (or its next chunk) over expanded keys and values
            (``mkv_latent_prefill``)
  tree      attention of a tree of drafted tokens over an FP16 cache (``mkv_tree_attention``)
  commit    the accepted path of a tree joins the cache (``mkv_tree_commit``, ``mkv_latent_commit``)

``own = False`` computes them with elementary torch operations in 32 bits; ``own = True`` calls the library.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
ROPE = 64          # rotated dimensions of a latent row


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # a chat's first replies: one token of one conversation, an odd length; latency counts
        dict(name="latent_token_short", op="latent", dtype="bf16", B=1, H=32, rank=512, n=1, T=777, tree=False,
             ragged=False),
        # the batch and context of the library's own decode benchmark, one token an entry
        dict(name="latent_token_batch", op="latent", dtype="fp16", B=8, H=32, rank=512, n=1, T=8192, tree=False,
             ragged=False),
        # verification of twelve drafted tokens an entry over long, unequal contexts
        dict(name="latent_tree_long", op="latent", dtype="bf16", B=4, H=32, rank=512, n=12, T=32768, tree=True,
             ragged=True),
        # the queries of a decode step carried into the latent space
        dict(name="absorb_token_batch", op="product", kind="absorb", dtype="fp16", B=8, H=32, rank=512, nope=128,
             vdim=128, n=1, T=0),
        # the outputs of a tree of drafted tokens carried out of it
        dict(name="project_tree", op="product", kind="project", dtype="bf16", B=4, H=32, rank=512, nope=128,
             vdim=128, n=12, T=0),
        # a whole prompt's rows expanded into keys and values
        dict(name="expand_prompt", op="product", kind="expand", dtype="fp16", B=1, H=32, rank=512, nope=128,
             vdim=128, n=1, T=8192),
        # a few short prompts of unequal, odd lengths
        dict(name="prefill_prompt_odd", op="prefill", dtype="bf16", B=3, H=32, nope=128, vdim=128, n=333, T=333,
             ragged=True),
        # the second half of an 8K prompt, attending to the first half already in the cache
        dict(name="prefill_chunk_long", op="prefill", dtype="fp16", B=1, H=32, nope=128, vdim=128, n=4096, T=8192,
             ragged=False),
        # a short chain of drafted tokens in one conversation; latency counts
        dict(name="tree_token_short", op="tree", B=1, Hq=32, Hkv=8, D=128, n=5, T=700, ragged=False),
        # sixteen drafted tokens an entry at the library's benchmark batch and context
        dict(name="tree_batch", op="tree", B=8, Hq=32, Hkv=8, D=128, n=16, T=8192, ragged=False),
        # the accepted paths of that tree join its FP16 caches
        dict(name="commit_fp16", op="commit", kind="fp16", dtype="fp16", B=8, Hkv=8, D=128, rank=0, n=16, T=8192),
        # and of a larger batch with latent caches
        dict(name="commit_latent", op="commit", kind="latent", dtype="bf16", B=16, Hkv=1, D=0, rank=512, n=33,
             T=4096),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["latent", "latent", "product", "prefill", "tree", "tree", "commit"])
    dtype = rng.choice(["fp16", "bf16"])
    H = rng.choice([8, 16, 20, 32, 64, 128])
    rank = rng.choice([256, 512, 512])
    nope, vdim = rng.choice([64, 128]), rng.choice([64, 128])
    if op == "latent":
        tree = rng.random() < 0.5
        n = _log(rng, 1, 64) if tree else 1
        B = _log(rng, 1, 16)
        T = _log(rng, 33, 32768)
        while B * T * n * H > 4 * 32768 * 12 * 32 or B * T > 8 * 32768:   # within the largest listed case's work
            T = max(1, T // 2)
        return dict(op="latent", dtype=dtype, B=B, H=H, rank=rank, n=n, T=T, tree=tree, ragged=rng.random() < 0.5)
    if op == "product":
        kind = rng.choice(["absorb", "project", "expand"])
        B = _log(rng, 1, 16)
        n = 1 if kind == "expand" else _log(rng, 1, 64)
        T = _log(rng, 33, 8192) // B + 1 if kind == "expand" else 0
        if kind == "expand":
            H = min(H, 32)
        return dict(op="product", kind=kind, dtype=dtype, B=B, H=H, rank=rank, nope=nope, vdim=vdim, n=n, T=T)
    if op == "prefill":
        B = _log(rng, 1, 8)
        n = _log(rng, 1, 4096)
        T = n + (_log(rng, 1, 4096) if rng.random() < 0.5 else 0)
        H = rng.choice([8, 16, 20, 32])
        while B * H * n * T > 32 * 4096 * 8192 * 3 // 4:
            n, T = max(1, n // 2), max(1, T // 2)
        return dict(op="prefill", dtype=dtype, B=B, H=H, nope=nope, vdim=vdim, n=n, T=max(T, n),
                    ragged=rng.random() < 0.5)
    if op == "tree":
        Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
        n, B, T = _log(rng, 1, 64), _log(rng, 1, 16), _log(rng, 33, 32768)
        while B * T * Hkv > 8 * 8192 * 8 or B * T * Hkv * G * n > 8 * 8192 * 32 * 48:
            T = max(1, T // 2)
        return dict(op="tree", B=B, Hq=Hkv * G, Hkv=Hkv, D=rng.choice([64, 128]), n=n, T=T,
                    ragged=rng.random() < 0.5)
    kind = rng.choice(["fp16", "latent"])
    n, B, T = _log(rng, 1, 64), _log(rng, 1, 16), _log(rng, 33, 8192)
    if kind == "fp16":
        return dict(op="commit", kind=kind, dtype="fp16", B=B, Hkv=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128]),
                    rank=0, n=n, T=T)
    return dict(op="commit", kind=kind, dtype=dtype, B=B, Hkv=1, D=0, rank=rank, n=n, T=T)


def _lengths(c):
    """Cached tokens of each entry: all T, or (ragged) unequal ones from T down to about T / 2."""
    B, T = c["B"], c["T"]
    return [T - (b * T) // (2 * B) for b in range(B)] if c.get("ragged") else [T] * B


def _query_lengths(c):
    """New tokens of each entry of a prefill: never more than it holds."""
    return [min(c["n"] - (b * c["n"]) // (2 * c["B"]) if c["ragged"] else c["n"], t)
            for b, t in enumerate(_lengths(c))]


def work(c):
    """What one pass cannot do without: each input read once, each output written once, each visible pair."""
    if c["op"] == "latent":
        row, R = c["rank"] + ROPE, c["n"] * c["H"]
        keys = sum(_lengths(c))
        vis = keys + (c["B"] * (c["n"] + 1) / 2 if c["tree"] else 0)
        return {"bytes": 2 * (keys * row + (c["B"] * c["n"] * row if c["tree"] else 0)
                              + c["B"] * R * (row + c["rank"])),
                "flops": 2 * R * vis * (row + c["rank"])}
    if c["op"] == "product":
        H, r, rows = c["H"], c["rank"], c["B"] * c["n"]
        if c["kind"] == "absorb":
            return {"bytes": 2 * (H * c["nope"] * r + rows * H * (c["nope"] + r + 2 * ROPE)),
                    "flops": 2 * rows * H * c["nope"] * r}
        if c["kind"] == "project":
            return {"bytes": 2 * (H * c["vdim"] * r + rows * H * (c["vdim"] + r)),
                    "flops": 2 * rows * H * c["vdim"] * r}
        tok, d = c["B"] * c["T"], c["nope"] + c["vdim"]
        return {"bytes": 2 * (H * d * r + tok * r + tok * H * d), "flops": 2 * tok * H * d * r}
    if c["op"] == "prefill":
        H, dk, dv = c["H"], c["nope"] + ROPE, c["vdim"]
        lens, qs = _lengths(c), _query_lengths(c)
        pairs = sum(q * (t - q) + q * (q + 1) / 2 for t, q in zip(lens, qs))
        return {"bytes": 2 * (sum(lens) * (H * (c["nope"] + dv) + ROPE) + sum(qs) * H * (dk + dv)),
                "flops": 2 * H * pairs * (dk + dv)}
    if c["op"] == "tree":
        keys = sum(_lengths(c))
        return {"bytes": 2 * c["D"] * (2 * c["Hkv"] * (keys + c["B"] * c["n"]) + 2 * c["B"] * c["n"] * c["Hq"]),
                "flops": 4 * c["D"] * c["Hq"] * c["n"] * (keys + c["B"] * (c["n"] + 1) / 2)}
    row = 2 * c["Hkv"] * c["D"] if c["kind"] == "fp16" else c["rank"] + ROPE
    moved = sum(_accepted(c))
    return {"bytes": 2 * 2 * row * moved + 4 * (moved + 3 * c["B"]), "flops": 0}


def _accepted(c):
    """Length of the accepted path of each entry, from none to all n."""
    return [((b * 7 + 3) % (c["n"] + 1)) for b in range(c["B"])]


# ------------------------------------------------------------------------------------------------ the inputs
def _tree_masks(B, n, seed):
    """A random tree an entry: token j's parent is an earlier one or the root; a token sees itself and its ancestors."""
    rng = np.random.default_rng(seed)
    masks = np.zeros((B, n), dtype=np.uint64)
    for j in range(n):
        parent = rng.integers(-1, j, size=B, endpoint=False) if j else np.full(B, -1)
        up = np.where(parent >= 0, masks[np.arange(B), np.maximum(parent, 0)], np.uint64(0))
        masks[:, j] = up | np.uint64(1 << j)
    return masks.view(np.int64)


def _case_dims(c):
    return dict(rank=c.get("rank", 512) or 512, nope=c.get("nope", 128), vdim=c.get("vdim", 128))


def prepare(c, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[c.get("dtype", "fp16")]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device=dev, dtype=torch.float32).mul_(std).to(dt)

    s = dict(c)
    B, n, T = c["B"], c["n"], c["T"]
    if c["op"] == "latent":
        row = c["rank"] + ROPE
        s["q"] = normal(B, n, c["H"], row)
        s["rows"] = normal(B, T + n, row)
        s["T_len"] = torch.tensor(_lengths(c), dtype=torch.int32, device=dev)
        s["new"] = normal(B, n, row) if c["tree"] else None
        s["mask"] = torch.from_numpy(_tree_masks(B, n, seed)).to(dev) if c["tree"] else None
        s["out"] = torch.empty(B, n, c["H"], c["rank"], dtype=dt, device=dev)
        s["scale"] = 1.0 / math.sqrt(128 + ROPE)
    elif c["op"] == "product":
        H, r = c["H"], c["rank"]
        s["w"] = normal(H, c["nope"] + c["vdim"], r, std=r ** -0.5)
        if c["kind"] == "absorb":
            s["x"] = normal(B, n, H, c["nope"] + ROPE)
            s["out"] = torch.empty(B, n, H, r + ROPE, dtype=dt, device=dev)
        elif c["kind"] == "project":
            s["x"] = normal(B, n, H, r)
            s["out"] = torch.empty(B, n, H, c["vdim"], dtype=dt, device=dev)
        else:
            s["x"] = normal(B, T, r + ROPE)
            s["T_len"] = torch.full((B,), T, dtype=torch.int32, device=dev)
            s["out"] = torch.empty(B, H, T, c["nope"] + c["vdim"], dtype=dt, device=dev)
    elif c["op"] == "prefill":
        H = c["H"]
        s["q"] = normal(B, n, H, c["nope"] + ROPE)
        s["kv"] = normal(B, H, T, c["nope"] + c["vdim"])
        s["rows"] = normal(B, T, 512 + ROPE)
        s["T_len"] = torch.tensor(_lengths(c), dtype=torch.int32, device=dev)
        s["q_len"] = torch.tensor(_query_lengths(c), dtype=torch.int32, device=dev)
        s["out"] = torch.empty(B, n, H, c["vdim"], dtype=dt, device=dev)
        s["scale"] = 1.0 / math.sqrt(c["nope"] + ROPE)
    elif c["op"] == "tree":
        s["q"] = normal(B, n, c["Hq"], c["D"])
        s["k"] = normal(B, c["Hkv"], T + n, c["D"])
        s["v"] = normal(B, c["Hkv"], T + n, c["D"])
        s["k_new"] = normal(B, n, c["Hkv"], c["D"])
        s["v_new"] = normal(B, n, c["Hkv"], c["D"])
        s["T_len"] = torch.tensor(_lengths(c), dtype=torch.int32, device=dev)
        s["mask"] = torch.from_numpy(_tree_masks(B, n, seed)).to(dev)
        s["out"] = torch.empty(B, n, c["Hq"], c["D"], dtype=dt, device=dev)
        s["scale"] = 1.0 / math.sqrt(c["D"])
    else:
        rng = np.random.default_rng(seed)
        path = np.sort(np.argsort(rng.random((B, n)), axis=1), axis=1)
        acc = _accepted(c)
        for b in range(B):     # a path's tokens in ascending order, then what a verifier leaves behind them
            path[b, :acc[b]] = np.sort(rng.permutation(n)[:acc[b]])
        s["path"] = torch.from_numpy(path.astype(np.int32)).to(dev)
        s["n_path"] = torch.tensor(acc, dtype=torch.int32, device=dev)
        s["T_before"] = torch.tensor([T - (b * T) // (2 * B) for b in range(B)], dtype=torch.int32, device=dev)
        s["T_len"] = s["T_before"].clone()
        if c["kind"] == "fp16":
            s["k"] = normal(B, c["Hkv"], T + n, c["D"])
            s["v"] = normal(B, c["Hkv"], T + n, c["D"])
            s["k_new"] = normal(B, n, c["Hkv"], c["D"])
            s["v_new"] = normal(B, n, c["Hkv"], c["D"])
        else:
            s["rows"] = normal(B, T + n, c["rank"] + ROPE)
            s["new"] = normal(B, n, c["rank"] + ROPE)
    if own:
        s["plan"] = _plan(c, s)
    return s


def _plan(c, s):
    """What a program that uses the library keeps beside its tensors: the configuration, the cache's struct, a workspace."""
    import paper_2609_07966_gb300 as mkv
    from paper_2609_07966_gb300 import caches
    p = {"mkv": mkv}
    if c["op"] == "tree" or (c["op"] == "commit" and c["kind"] == "fp16"):
        p["cfg"] = mkv.config(mkv.MKV_FP16, c["B"], c.get("Hq", c["Hkv"]), c["Hkv"], c["D"])
        p["cache"] = caches.wrap_cache(p["cfg"], s["T_len"], s["k"], s["v"])
        if c["op"] == "tree":
            p["ws"], p["ws_bytes"] = caches.tree_workspace(p["cfg"], c["T"] + c["n"], c["n"])
        return p
    dims = _case_dims(c)
    p["cfg"] = mkv.latent_config(mkv.MKV_BF16 if c["dtype"] == "bf16" else mkv.MKV_F16, c["B"], c.get("H", 1),
                                 rank=dims["rank"], rope_dim=ROPE, nope_dim=dims["nope"], v_dim=dims["vdim"])
    rows = s["x"] if c["op"] == "product" and c["kind"] == "expand" else s.get("rows")
    if rows is not None:
        p["cache"] = caches.wrap_latent_cache(p["cfg"], s["T_len"], rows)
    if c["op"] == "latent":
        p["ws"], p["ws_bytes"] = caches.latent_workspace(p["cfg"], c["T"] + c["n"], c["n"])
    return p


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return _own(s) if own else _PLAIN[s["op"]](s)


def _own(s):
    p = s["plan"]
    mkv, cfg = p["mkv"], p["cfg"]
    if s["op"] == "latent":
        tree = s["tree"]
        mkv.mkv_latent_attention(cfg, s["q"].data_ptr(), p["cache"].c, s["new"].data_ptr() if tree else 0,
                                 s["mask"].data_ptr() if tree else 0, s["n"], s["out"].data_ptr(), p["ws"].data_ptr(),
                                 p["ws_bytes"])
        return {"out": s["out"]}
    if s["op"] == "product":
        if s["kind"] == "absorb":
            mkv.mkv_latent_absorb(cfg, s["x"].data_ptr(), s["w"].data_ptr(), s["n"], s["out"].data_ptr())
        elif s["kind"] == "project":
            mkv.mkv_latent_project(cfg, s["x"].data_ptr(), s["w"].data_ptr(), s["n"], s["out"].data_ptr())
        else:
            mkv.mkv_latent_expand(cfg, p["cache"].c, s["w"].data_ptr(), s["T"], s["out"].data_ptr())
        return {"out": s["out"]}
    if s["op"] == "prefill":
        mkv.mkv_latent_prefill(cfg, s["q"].data_ptr(), s["kv"].data_ptr(), s["T"], p["cache"].c,
                               s["q_len"].data_ptr(), s["n"], s["out"].data_ptr())
        return {"out": s["out"]}
    if s["op"] == "tree":
        mkv.mkv_tree_attention(cfg, s["q"].data_ptr(), p["cache"].c, s["k_new"].data_ptr(), s["v_new"].data_ptr(),
                               s["mask"].data_ptr(), s["n"], s["out"].data_ptr(), p["ws"].data_ptr(), p["ws_bytes"])
        return {"out": s["out"]}
    s["T_len"].copy_(s["T_before"])       # the lengths before the step, so that a pass can be repeated
    if s["kind"] == "fp16":
        mkv.mkv_tree_commit(cfg, s["k_new"].data_ptr(), s["v_new"].data_ptr(), s["path"].data_ptr(),
                            s["n_path"].data_ptr(), s["n"], p["cache"].c)
        return {"k": s["k"], "v": s["v"], "T_len": s["T_len"]}
    mkv.mkv_latent_commit(cfg, s["new"].data_ptr(), s["path"].data_ptr(), s["n_path"].data_ptr(), s["n"],
                          p["cache"].c)
    return {"rows": s["rows"], "T_len": s["T_len"]}


def _attend(scores, visible, values):
    """softmax over the visible keys (a row that sees none gives zeros) times the values, all in 32 bits."""
    low = torch.where(visible, scores, torch.full_like(scores, -3.0e38))
    e = torch.exp(low - low.amax(-1, keepdim=True)) * visible
    total = e.sum(-1, keepdim=True)
    return (e @ values) / torch.where(total > 0, total, torch.ones_like(total))


def _tree_visible(mask, n):
    """[B][n][n]: query i sees drafted token j."""
    j = torch.arange(n, device=mask.device)
    return ((mask[:, :, None] >> j) & 1).bool()


def _plain_latent(s):
    B, n, H, r = s["B"], s["n"], s["H"], s["rank"]
    cap = s["rows"].shape[1]
    q = s["q"].float().reshape(B, n * H, -1)
    rows = s["rows"].float()
    vis = (torch.arange(cap, device=q.device) < s["T_len"][:, None])[:, None, :].expand(B, n, cap)
    if s["tree"]:
        rows = torch.cat([rows, s["new"].float()], 1)
        vis = torch.cat([vis, _tree_visible(s["mask"], n)], 2)
    vis = vis[:, :, None, :].expand(B, n, H, vis.shape[-1]).reshape(B, n * H, -1)
    o = _attend((q @ rows.transpose(1, 2)) * s["scale"], vis, rows[..., :r])
    return {"out": o.reshape(B, n, H, r).to(s["q"].dtype)}


def _plain_product(s):
    x, w = s["x"].float(), s["w"].float()
    if s["kind"] == "absorb":
        up = torch.einsum("bihd,hdr->bihr", x[..., :s["nope"]], w[:, :s["nope"]])
        o = torch.cat([up, x[..., s["nope"]:]], -1)
    elif s["kind"] == "project":
        o = torch.einsum("bihr,hdr->bihd", x, w[:, s["nope"]:])
    else:
        o = torch.einsum("btr,hdr->bhtd", x[..., :s["rank"]], w)
    return {"out": o.to(s["x"].dtype)}


def _plain_prefill(s):
    n, T, d = s["n"], s["T"], s["nope"]
    q = s["q"].float().transpose(1, 2)
    kv, rope = s["kv"].float(), s["rows"].float()[:, :, 512:]
    sc = q[..., :d] @ kv[..., :d].transpose(2, 3) + q[..., d:] @ rope[:, None].transpose(2, 3)
    i = torch.arange(n, device=q.device)
    pos = torch.where(i < s["q_len"][:, None], s["T_len"][:, None] - s["q_len"][:, None] + i, -1)
    vis = torch.arange(T, device=q.device) <= pos[:, None, :, None]
    return {"out": _attend(sc * s["scale"], vis, kv[..., d:]).transpose(1, 2).to(s["q"].dtype)}


def _plain_tree(s):
    B, n, Hq, Hkv, D = s["B"], s["n"], s["Hq"], s["Hkv"], s["D"]
    G, cap = Hq // Hkv, s["k"].shape[2]
    q = s["q"].float().reshape(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    k = torch.cat([s["k"].float(), s["k_new"].float().transpose(1, 2)], 2)
    v = torch.cat([s["v"].float(), s["v_new"].float().transpose(1, 2)], 2)
    vis = (torch.arange(cap, device=q.device) < s["T_len"][:, None])[:, None, :].expand(B, n, cap)
    vis = torch.cat([vis, _tree_visible(s["mask"], n)], 2)[:, None, :, None, :]
    vis = vis.expand(B, Hkv, n, G, cap + n).reshape(B, Hkv, n * G, cap + n)
    o = _attend((q @ k.transpose(2, 3)) * s["scale"], vis, v)
    return {"out": o.reshape(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D).to(s["q"].dtype)}


def _plain_commit(s):
    B, n = s["B"], s["n"]
    i = torch.arange(n, device=s["path"].device)
    b = torch.arange(B, device=i.device)[:, None]
    dst = (s["T_before"][:, None] + i).long()                    # [B][n]
    taken = (i < s["n_path"][:, None])
    src = s["path"].long()

    def place(cache, new):                                       # cache [B][slots][...], new [B][n][...]
        keep = taken.reshape(B, n, *([1] * (new.dim() - 2)))
        cache[b, dst] = torch.where(keep, new[b, src], cache[b, dst])

    s["T_len"].copy_(s["T_before"] + s["n_path"])
    if s["kind"] == "fp16":
        place(s["k"].transpose(1, 2), s["k_new"])
        place(s["v"].transpose(1, 2), s["v_new"])
        return {"k": s["k"], "v": s["v"], "T_len": s["T_len"]}
    place(s["rows"], s["new"])
    return {"rows": s["rows"], "T_len": s["T_len"]}


_PLAIN = {"latent": _plain_latent, "product": _plain_product, "prefill": _plain_prefill, "tree": _plain_tree,
          "commit": _plain_commit}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(c, seed):
    """The definitions in 64 bits, entry by entry and over the visible tokens alone (commit moves rows: no value)."""
    if c["op"] == "commit":
        return None
    s = prepare(c, seed)
    if c["op"] == "product":
        return {"out": _exact_product(c, s)}
    return {"out": {"latent": _exact_latent, "prefill": _exact_prefill, "tree": _exact_tree}[c["op"]](c, s)}


def _exact_softmax(logits):
    z = logits - logits.max(dim=-1, keepdim=True).values
    z = z.exp()
    return z / z.sum(dim=-1, keepdim=True)


def _exact_latent(c, s):
    out = torch.zeros(c["B"], c["n"], c["H"], c["rank"], dtype=torch.float64, device="cuda")
    for b, t in enumerate(_lengths(c)):
        for i in range(c["n"]):
            seen = s["rows"][b, :t].double()
            if c["tree"]:
                bits = int(s["mask"][b, i]) & ((1 << 64) - 1)
                picks = [j for j in range(c["n"]) if bits >> j & 1]
                seen = torch.cat([seen, s["new"][b, picks].double()])
            p = _exact_softmax(torch.matmul(s["q"][b, i].double(), seen.T) * s["scale"])
            out[b, i] = torch.matmul(p, seen[:, :c["rank"]])
    return out


def _exact_product(c, s):
    x, w = s["x"].double(), s["w"].double()
    if c["kind"] == "expand":
        return torch.stack([torch.stack([x[b, :, :c["rank"]] @ w[h].T for h in range(c["H"])])
                            for b in range(c["B"])])
    heads = []
    for h in range(c["H"]):
        if c["kind"] == "absorb":
            heads.append(torch.cat([x[:, :, h, :c["nope"]] @ w[h, :c["nope"]], x[:, :, h, c["nope"]:]], -1))
        else:
            heads.append(x[:, :, h] @ w[h, c["nope"]:].T)
    return torch.stack(heads, 2)


def _exact_prefill(c, s):
    out = torch.zeros(c["B"], c["n"], c["H"], c["vdim"], dtype=torch.float64, device="cuda")
    for b, (t, m) in enumerate(zip(_lengths(c), _query_lengths(c))):
        later = torch.ones(m, t, dtype=torch.bool, device="cuda").triu(t - m + 1)
        for h in range(c["H"]):
            keys = torch.cat([s["kv"][b, h, :t, :c["nope"]], s["rows"][b, :t, 512:]], -1).double()
            logits = s["q"][b, :m, h].double() @ keys.T * s["scale"]
            out[b, :m, h] = _exact_softmax(logits.masked_fill(later, -math.inf)) @ s["kv"][b, h, :t, c["nope"]:].double()
    return out


def _exact_tree(c, s):
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros(c["B"], c["n"], c["Hq"], c["D"], dtype=torch.float64, device="cuda")
    for b, t in enumerate(_lengths(c)):
        k, v = s["k"][b, :, :t].double(), s["v"][b, :, :t].double()
        for i in range(c["n"]):
            bits = int(s["mask"][b, i]) & ((1 << 64) - 1)
            picks = [j for j in range(c["n"]) if bits >> j & 1]
            ki = torch.cat([k, s["k_new"][b, picks].double().transpose(0, 1)], 1)
            vi = torch.cat([v, s["v_new"][b, picks].double().transpose(0, 1)], 1)
            p = _exact_softmax(s["q"][b, i].double().reshape(c["Hkv"], G, -1) @ ki.transpose(1, 2) * s["scale"])
            out[b, i] = (p @ vi).reshape(c["Hq"], -1)
    return out

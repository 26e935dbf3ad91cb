"""GPU parity of latent attention: products, absorbed and expanded attention, commit."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import latent as L
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import check_attention, check_product, f64, randn, to_mask, torch_dtype, tree_masks

pytestmark = pytest.mark.gpu

KINDS = {"fp16": mkv.MKV_F16, "bf16": mkv.MKV_BF16}


# ------------------------------------------------------------------------------------------- absorbed attention
def _case(dtype, B, H, rank, n, T_cap, lens, seed, tree=True, masks=None, junk=None):
    torch = torch_cuda()
    rng = np.random.default_rng(seed)
    row = rank + 64
    c = dict(dtype=dtype, B=B, H=H, rank=rank, n=n, lens=lens, tree=tree)
    c["cfg"] = mkv.latent_config(KINDS[dtype], B, H, rank=rank)
    c["q"] = randn(rng, (B, n, H, row), dtype)
    c["rows"] = randn(rng, (B, T_cap, row), dtype)
    c["new"] = randn(rng, (B, n, row), dtype)
    if junk is not None:
        for b, t in enumerate(lens):
            c["rows"][b, t:] = junk
    c["mask"] = tree_masks(rng, B, n) if masks is None else masks
    c["cache"] = caches.wrap_latent_cache(c["cfg"], torch.tensor(lens, dtype=torch.int32, device="cuda"), c["rows"])
    return c


def _run(c, stream=None):
    torch = torch_cuda()
    ws, nws = caches.latent_workspace(c["cfg"], c["cache"].T_cap, c["n"])
    ws.fill_(255)
    ws[:16384] = 0
    out = torch.full((c["B"], c["n"], c["H"], c["rank"]), float("nan"), dtype=c["q"].dtype, device="cuda")
    m = to_mask(c["mask"])
    torch.cuda.synchronize()
    mkv.mkv_latent_attention(c["cfg"], c["q"].data_ptr(), c["cache"].c, c["new"].data_ptr() if c["tree"] else 0,
                             m.data_ptr() if c["tree"] else 0, c["n"], out.data_ptr(), ws.data_ptr(), nws, stream)
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == 0
    return out


def _check(c, out, what=""):
    n, H, r = c["n"], c["H"], c["rank"]
    for b, t in enumerate(c["lens"]):
        keys = f64(c["rows"][b, :t])
        if c["tree"]:
            keys = np.concatenate([keys, f64(c["new"][b])])
            vis = L.tree_visible(c["mask"][b], n, t)
        else:
            vis = np.ones((n, t), bool)
        ref, mag = L.attend_visible(f64(c["q"][b]).reshape(n * H, -1), keys, keys[:, :r], np.repeat(vis, H, axis=0),
                                    (128 + 64) ** -0.5)
        check_attention(out[b].reshape(n * H, r), ref, mag, c["dtype"], f"{what} b{b}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rank", [256, 512])
@pytest.mark.parametrize("H,n,tree", [(1, 1, False), (8, 1, False), (20, 3, True), (32, 1, True), (128, 1, False),
                                      (16, 64, True), (48, 5, False)])
def test_absorbed_shapes(dtype, rank, H, n, tree):
    lens = [0, 1, 63, 64, 65, 333]
    c = _case(dtype, len(lens), H, rank, n, 384, lens, seed=rank + H + n, tree=tree, junk=float("nan"))
    _check(c, _run(c), f"{dtype} r{rank} H{H} n{n}")


@pytest.mark.parametrize("T", [1000, 8192, 30011])
def test_absorbed_long_contexts_split(T):
    c = _case("fp16", 2, 16, 512, 2, T + 1, [T, T // 2 + 1], seed=T)
    _check(c, _run(c), f"T{T}")


@pytest.mark.parametrize("H,n,tree", [(8, 1, False), (32, 5, True)])
def test_absorbed_many_ragged_units(H, n, tree):
    """More units than SMs, of unequal lengths: runs of tiles that hold whole units and parts of others; then all empty."""
    lens = [(29 * b * b) % 300 if b % 5 else 0 for b in range(80)]
    c = _case("bf16", 80, H, 256, n, 320, lens, seed=H, tree=tree, junk=float("nan"))
    _check(c, _run(c), f"H{H} n{n}")
    c["cache"].t["T_len"].zero_()
    c["lens"] = [0] * 80
    out = _run(c)
    if tree:
        _check(c, out, "empty cache")
    else:
        assert (f64(out) == 0).all()


def test_absorbed_empty_rows_are_zero():
    masks = np.array([[0b10, 0, 0b100]], dtype=np.uint64)
    c = _case("bf16", 1, 8, 512, 3, 64, [0], seed=2, masks=masks, junk=float("nan"))
    out = _run(c)
    assert (f64(out[0, 1]) == 0).all()
    _check(c, out, "empty")
    c = _case("fp16", 2, 8, 256, 2, 64, [0, 0], seed=2, tree=False, junk=float("inf"))
    assert (f64(_run(c)) == 0).all()


@pytest.mark.parametrize("rank", [256, 512])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_absorbed_unseen_tokens_do_not_leak(rank, bad):
    masks = np.array([[0b001, 0b011, 0b101]], dtype=np.uint64)
    for t in (0, 70):
        c = _case("bf16", 1, 4, rank, 3, 128, [t], seed=5, masks=masks)
        c["new"][0, 1, 9] = bad                       # a latent value: part of the key and of the value
        out = f64(_run(c))
        assert np.isfinite(out[0, [0, 2]]).all() and not np.isfinite(out[0, 1]).all()
        c["q"], c["new"] = c["q"][:, [0, 2]].contiguous(), c["new"][:, [0, 2]].contiguous()
        c["n"], c["mask"] = 2, np.array([[0b01, 0b11]], dtype=np.uint64)
        import torch
        _check(c, torch.from_numpy(out[:, [0, 2]]), "others")


def test_absorbed_growing_scores_and_streams():
    import torch
    c = _case("fp16", 2, 32, 512, 4, 3000, [2990, 1234], seed=9)
    ramp = torch.linspace(0.02, 5.0, 3000, device="cuda")[None, :, None]
    c["rows"].copy_((c["rows"].float() * ramp).to(c["rows"].dtype))
    first = _run(c)
    _check(c, first, "ramp")
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        again = _run(c)
    assert torch.equal(first, again) and torch.equal(first, _run(c, st.cuda_stream))


def test_absorbed_offsets_past_32_bits():
    import torch
    torch_cuda()
    T_cap, T = 4_200_000, 4_199_999                  # 4.8 GB an entry
    cfg = mkv.latent_config(mkv.MKV_F16, 1, 4)
    rows = torch.zeros((1, T_cap, 576), dtype=torch.float16, device="cuda")
    rows[0, T - 1, 575] = 60.0
    rows[0, T - 1, :512] = torch.arange(512, device="cuda").to(torch.float16) / 16
    q = torch.zeros((1, 1, 4, 576), dtype=torch.float16, device="cuda")
    q[..., 575] = 60.0
    cache = caches.wrap_latent_cache(cfg, torch.tensor([T], dtype=torch.int32, device="cuda"), rows)
    ws, nws = caches.latent_workspace(cfg, T_cap, 1)
    out = torch.full((1, 1, 4, 512), float("nan"), dtype=torch.float16, device="cuda")
    mkv.mkv_latent_attention(cfg, q.data_ptr(), cache.c, 0, 0, 1, out.data_ptr(), ws.data_ptr(), nws)
    assert mkv.mkv_get_status() == 0
    np.testing.assert_allclose(f64(out[0, 0]), np.tile(np.arange(512) / 16, (4, 1)), rtol=1e-3)


# ------------------------------------------------------------------------------------------- products
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("nope,vdim,rank", [(128, 128, 512), (64, 128, 256), (128, 64, 512), (64, 64, 512)])
@pytest.mark.parametrize("B,n,H", [(1, 1, 1), (3, 5, 7), (2, 64, 4), (1, 200, 2)])
def test_absorb_and_project(dtype, nope, vdim, rank, B, n, H):
    torch = torch_cuda()
    rng = np.random.default_rng(nope + vdim + n)
    cfg = mkv.latent_config(KINDS[dtype], B, H, rank=rank, nope_dim=nope, v_dim=vdim)
    w = randn(rng, (H, nope + vdim, rank), dtype, std=rank ** -0.5)
    q = randn(rng, (B, n, H, nope + 64), dtype)
    o = randn(rng, (B, n, H, rank), dtype)
    qa = torch.full((B, n, H, rank + 64), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    out = torch.full((B, n, H, vdim), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    mkv.mkv_latent_absorb(cfg, q.data_ptr(), w.data_ptr(), n, qa.data_ptr())
    mkv.mkv_latent_project(cfg, o.data_ptr(), w.data_ptr(), n, out.data_ptr())
    assert mkv.mkv_get_status() == 0
    w64, q64, o64 = f64(w), f64(q).reshape(B * n, H, -1), f64(o).reshape(B * n, H, -1)
    check_product(qa.reshape(B * n, H, -1), L.absorb(q64, w64[:, :nope], nope),
                  L.absorb(np.abs(q64), np.abs(w64[:, :nope]), nope), dtype, "absorb")
    assert torch.equal(qa[..., rank:], q[..., nope:])
    check_product(out.reshape(B * n, H, -1), L.project(o64, w64[:, nope:]),
                  L.project(np.abs(o64), np.abs(w64[:, nope:])), dtype, "project")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("nope,vdim,rank", [(128, 128, 512), (64, 128, 256), (128, 64, 512), (64, 64, 256)])
@pytest.mark.parametrize("T_max,lens", [(1, [1, 0]), (130, [130, 77]), (333, [400, 129])])
def test_expand(dtype, nope, vdim, rank, T_max, lens):
    torch = torch_cuda()
    rng = np.random.default_rng(nope + vdim + T_max)
    B, H, T_cap = len(lens), 3, 400
    cfg = mkv.latent_config(KINDS[dtype], B, H, rank=rank, nope_dim=nope, v_dim=vdim)
    w = randn(rng, (H, nope + vdim, rank), dtype, std=rank ** -0.5)
    rows = randn(rng, (B, T_cap, rank + 64), dtype)
    cache = caches.wrap_latent_cache(cfg, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows)
    kv = torch.full((B, H, T_max, nope + vdim), 7.0, dtype=torch_dtype(dtype), device="cuda")
    mkv.mkv_latent_expand(cfg, cache.c, w.data_ptr(), T_max, kv.data_ptr())
    assert mkv.mkv_get_status() == 0
    for b, t in enumerate(lens):
        t = min(t, T_max)
        c, w64 = f64(rows[b, :t, :rank]), f64(w)
        check_product(kv[b, :, :t], L.expand(c, w64), L.expand(np.abs(c), np.abs(w64)), dtype, f"b{b}")
        assert (kv[b, :, t:] == 7.0).all(), "rows past the length are not written"


# ------------------------------------------------------------------------------------------- expanded attention
def _prefill(dtype, nope, vdim, H, n, T_max, lens, qlens, seed, junk=None, edit=None):
    torch = torch_cuda()
    rng = np.random.default_rng(seed)
    B, T_cap, rank = len(lens), T_max + 3, 256
    cfg = mkv.latent_config(KINDS[dtype], B, H, rank=rank, nope_dim=nope, v_dim=vdim)
    q = randn(rng, (B, n, H, nope + 64), dtype)
    kv = randn(rng, (B, H, T_max, nope + vdim), dtype)
    rows = randn(rng, (B, T_cap, rank + 64), dtype)
    if junk is not None:
        for b, t in enumerate(lens):
            kv[b, :, t:] = junk
            rows[b, t:] = junk
    if edit is not None:
        edit(q, kv, rows)
    cache = caches.wrap_latent_cache(cfg, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows)
    out = torch.full((B, n, H, vdim), float("nan"), dtype=torch_dtype(dtype), device="cuda")
    ql = None if qlens is None else torch.tensor(qlens, dtype=torch.int32, device="cuda")
    mkv.mkv_latent_prefill(cfg, q.data_ptr(), kv.data_ptr(), T_max, cache.c, 0 if ql is None else ql.data_ptr(), n,
                           out.data_ptr())
    assert mkv.mkv_get_status() == 0
    return q, kv, rows[..., rank:], out


def _check_prefill(r, dtype, nope, lens, qlens, what=""):
    q, kv, rope, out = r
    B, n, H = q.shape[:3]
    for b, t in enumerate(lens):
        ql = n if qlens is None else qlens[b]
        vis = L.causal_visible(ql, n, t)
        for h in range(H):
            K = np.concatenate([f64(kv[b, h, :t, :nope]), f64(rope[b, :t])], 1)
            ref, mag = L.attend_visible(f64(q[b, :, h]), K, f64(kv[b, h, :t, nope:]), vis, (nope + 64) ** -0.5)
            check_attention(out[b, :, h], ref, mag, dtype, f"{what} b{b} h{h}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("nope,vdim", [(128, 128), (64, 128), (128, 64), (64, 64)])
@pytest.mark.parametrize("n", [1, 127, 129, 300])
def test_prefill_shapes(dtype, nope, vdim, n):
    T_max = n + 130
    lens, qlens = [T_max, n, n // 2 + 1, 0], [n, n, n // 2 + 1, 0]
    r = _prefill(dtype, nope, vdim, 3, n, T_max, lens, qlens, seed=n + nope, junk=float("nan"))
    _check_prefill(r, dtype, nope, lens, qlens, f"n{n}")


def test_prefill_without_lengths_and_before_position_zero():
    lens = [40, 300, 513]
    r = _prefill("fp16", 128, 128, 2, 100, 513, lens, None, seed=1, junk=float("inf"))
    out = r[3]
    assert (f64(out[0, :60]) == 0).all(), "queries before position 0 see nothing"
    _check_prefill(r, "fp16", 128, lens, None)


def test_prefill_long_history_and_growing_scores():
    import torch
    T = 2500

    def grow(q, kv, rows):
        kv[..., :128] *= torch.linspace(0.05, 4.0, T, device="cuda")[None, None, :, None].to(kv.dtype)
    r = _prefill("bf16", 128, 128, 2, 260, T, [T, 1999], [260, 131], seed=3, edit=grow)
    _check_prefill(r, "bf16", 128, [T, 1999], [260, 131])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_prefill_later_tokens_do_not_leak(bad):
    """A token's non-finite values reach only the queries at or past it."""
    def edit(q, kv, rows):
        kv[0, 0, 200, 128 + 3] = bad                  # a value
        kv[0, 1, 150, 5] = bad                        # a key
    q, kv, rope, out = _prefill("fp16", 128, 128, 2, 300, 300, [300], None, seed=4, edit=edit)
    o = f64(out)
    assert np.isfinite(o[0, :200, 0]).all() and np.isfinite(o[0, :150, 1]).all()
    assert not np.isfinite(o[0, 200:, 0, 3]).any()
    assert np.isfinite(np.delete(o[0, 200:, 0], 3, axis=1)).all()
    vis = L.causal_visible(200, 200, 200)
    K = np.concatenate([f64(kv[0, 0, :200, :128]), f64(rope[0, :200])], 1)
    ref, mag = L.attend_visible(f64(q[0, :200, 0]), K, f64(kv[0, 0, :200, 128:]), vis, 192 ** -0.5)
    check_attention(out[0, :200, 0], ref, mag, "fp16", "before")


def test_expanded_and_absorbed_forms_agree():
    """The same attention both ways, each stage rounded to the type: within a few of its units."""
    torch = torch_cuda()
    rng = np.random.default_rng(12)
    B, H, T, n = 2, 8, 300, 4
    cfg = mkv.latent_config(mkv.MKV_F16, B, H)
    w = randn(rng, (H, 256, 512), "fp16", std=512 ** -0.5)
    rows = randn(rng, (B, T, 576), "fp16")
    q = randn(rng, (B, n, H, 192), "fp16")
    cache = caches.alloc_latent_cache(cfg, T)
    mkv.mkv_latent_commit(cfg, rows.data_ptr(), 0, 0, T, cache.c)
    kv = torch.zeros((B, H, T, 256), dtype=torch.float16, device="cuda")
    mkv.mkv_latent_expand(cfg, cache.c, w.data_ptr(), T, kv.data_ptr())
    full = torch.zeros((B, n, H, 128), dtype=torch.float16, device="cuda")
    mkv.mkv_latent_prefill(cfg, q.data_ptr(), kv.data_ptr(), T, cache.c, 0, n, full.data_ptr())
    # absorbed: the last n rows as a chain of drafted tokens over the others
    cache.t["T_len"].fill_(T - n)
    chain = np.array([[(1 << (i + 1)) - 1 for i in range(n)]] * B, dtype=np.uint64)
    qa = torch.zeros((B, n, H, 576), dtype=torch.float16, device="cuda")
    ol = torch.zeros((B, n, H, 512), dtype=torch.float16, device="cuda")
    out = torch.zeros_like(full)
    ws, nws = caches.latent_workspace(cfg, T, n)
    mkv.mkv_latent_absorb(cfg, q.data_ptr(), w.data_ptr(), n, qa.data_ptr())
    new, mask = rows[:, T - n:].contiguous(), to_mask(chain)
    mkv.mkv_latent_attention(cfg, qa.data_ptr(), cache.c, new.data_ptr(), mask.data_ptr(), n, ol.data_ptr(),
                             ws.data_ptr(), nws)
    mkv.mkv_latent_project(cfg, ol.data_ptr(), w.data_ptr(), n, out.data_ptr())
    assert mkv.mkv_get_status() == 0
    a, b = f64(full), f64(out)
    assert np.linalg.norm(a - b) <= 8 * 2.0 ** -11 * np.linalg.norm(a)


# ------------------------------------------------------------------------------------------- commit
@pytest.mark.parametrize("dtype,rank,n", [("fp16", 512, 1), ("bf16", 256, 33), ("fp16", 512, 700), ("bf16", 512, 2000)])
def test_latent_commit(dtype, rank, n):
    """Short paths go in one launch, a prompt's rows in two."""
    torch = torch_cuda()
    rng = np.random.default_rng(n)
    B, T_cap, lens = 3, 2500, [0, 800, 2499]
    cfg = mkv.latent_config(KINDS[dtype], B, 4, rank=rank)
    cache = caches.alloc_latent_cache(cfg, T_cap)
    cache.t["T_len"].copy_(torch.tensor(lens, dtype=torch.int32))
    new = randn(rng, (B, n, rank + 64), dtype)
    path = np.stack([rng.permutation(n) for _ in range(B)]).astype(np.int32)
    acc = [n, (n + 1) // 2, 1]
    ref = cache.t["rows"].clone()
    for b in range(B):
        ref[b, lens[b]:lens[b] + acc[b]] = new[b, torch.from_numpy(path[b, :acc[b]]).long().cuda()]
    path_d, acc_d = torch.from_numpy(path).cuda(), torch.tensor(acc, dtype=torch.int32, device="cuda")
    mkv.mkv_latent_commit(cfg, new.data_ptr(), path_d.data_ptr(), acc_d.data_ptr(), n, cache.c)
    assert mkv.mkv_get_status() == 0
    assert torch.equal(cache.t["rows"], ref)
    assert cache.t["T_len"].tolist() == [t + a for t, a in zip(lens, acc)]

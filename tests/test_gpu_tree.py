"""GPU parity of the tree operators: attention of drafted tokens over an FP16 cache, and the commit."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import latent as L
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import check_attention, f64, randn, to_mask, tree_masks

pytestmark = pytest.mark.gpu


def _case(B, Hkv, G, D, n, T_cap, lens, seed, masks=None, junk=None):
    """Inputs on the device; slots past an entry's length hold `junk`."""
    torch = torch_cuda()
    rng = np.random.default_rng(seed)
    c = dict(B=B, Hkv=Hkv, G=G, D=D, n=n, lens=lens)
    c["cfg"] = mkv.config(mkv.MKV_FP16, B, Hkv * G, Hkv, D)
    c["q"] = randn(rng, (B, n, Hkv * G, D), "fp16")
    c["k"], c["v"] = randn(rng, (B, Hkv, T_cap, D), "fp16"), randn(rng, (B, Hkv, T_cap, D), "fp16")
    c["kt"], c["vt"] = randn(rng, (B, n, Hkv, D), "fp16"), randn(rng, (B, n, Hkv, D), "fp16")
    if junk is not None:
        for b, t in enumerate(lens):
            c["k"][b, :, t:] = junk
            c["v"][b, :, t:] = junk
    c["mask"] = tree_masks(rng, B, n) if masks is None else masks
    c["cache"] = caches.wrap_cache(c["cfg"], torch.tensor(lens, dtype=torch.int32, device="cuda"), c["k"], c["v"])
    return c


def _run(c, stream=None):
    torch = torch_cuda()
    ws, nws = caches.tree_workspace(c["cfg"], c["cache"].T_cap, c["n"])
    ws.fill_(255)                       # a workspace's contents do not matter past its counters
    ws[:16384] = 0
    out = torch.full_like(c["q"], float("nan"))
    m = to_mask(c["mask"])
    torch.cuda.synchronize()
    mkv.mkv_tree_attention(c["cfg"], c["q"].data_ptr(), c["cache"].c, c["kt"].data_ptr(), c["vt"].data_ptr(),
                           m.data_ptr(), c["n"], out.data_ptr(), ws.data_ptr(), nws, stream)
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == 0
    return out


def _check(c, out, what="", entries=None):
    n, G, D = c["n"], c["G"], c["D"]
    for b in range(c["B"]) if entries is None else entries:
        t = c["lens"][b]
        vis = np.repeat(L.tree_visible(c["mask"][b], n, t), G, axis=0)
        for h in range(c["Hkv"]):
            q = f64(c["q"][b, :, h * G:(h + 1) * G]).reshape(n * G, D)
            K = np.concatenate([f64(c["k"][b, h, :t]), f64(c["kt"][b, :, h])])
            V = np.concatenate([f64(c["v"][b, h, :t]), f64(c["vt"][b, :, h])])
            ref, mag = L.attend_visible(q, K, V, vis, D ** -0.5)
            check_attention(out[b, :, h * G:(h + 1) * G].reshape(n * G, D), ref, mag, "fp16", f"{what} b{b} h{h}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("n", [1, 5, 33, 64])
def test_shapes(D, G, n):
    lens = [0, 1, 127, 128, 129, 700]
    c = _case(len(lens), 2, G, D, n, 768, lens, seed=D + 10 * G + 100 * n, junk=float("nan"))
    _check(c, _run(c), f"D{D} G{G} n{n}")


@pytest.mark.parametrize("T", [2048, 8191, 20000])
def test_long_contexts_split(T):
    """Few rows over a long context: the keys are split over many CTAs and joined."""
    c = _case(2, 2, 4, 128, 7, T + 16, [T, T // 3], seed=T)
    _check(c, _run(c), f"T{T}")


@pytest.mark.parametrize("Hkv,T,T_cap", [(8, 9001, 12000), (8, 100, 12000), (4, 7999, 8000), (2, 33000, 33008)])
def test_one_long_entry(Hkv, T, T_cap):
    """One entry alone, with capacity to spare: a key head's keys are split over a cluster or over runs."""
    c = _case(1, Hkv, 4, 128, 6, T_cap, [T], seed=T, junk=float("nan"))
    _check(c, _run(c), f"T{T} of {T_cap}")


@pytest.mark.parametrize("D", [64, 128])
def test_many_ragged_units(D):
    """More units than SMs, of unequal lengths, some empty: runs of tiles that hold whole units and parts of others."""
    lens = [(37 * b * b) % 500 if b % 7 else 0 for b in range(45)]
    c = _case(45, 4, 2, D, 3, 512, lens, seed=D, junk=float("nan"))
    _check(c, _run(c), f"D{D}", entries=range(0, 45, 4))


def test_empty_rows_are_zero():
    masks = np.array([[0, 0b10, 0], [0, 0, 0]], dtype=np.uint64)
    c = _case(2, 2, 4, 64, 3, 64, [0, 0], seed=3, masks=masks, junk=float("inf"))
    out = _run(c)
    assert (f64(out[0, 0]) == 0).all() and (f64(out[0, 2]) == 0).all() and (f64(out[1]) == 0).all()
    _check(c, out, "empty")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_unseen_tokens_do_not_leak(D, bad):
    """Token 2 holds non-finite keys and values; only the rows that see it may show it."""
    masks = np.array([[0b0001, 0b0011, 0b0101, 0b1001]], dtype=np.uint64)
    for t in (0, 130):
        c = _case(1, 2, 2, D, 4, 192, [t], seed=4, masks=masks)
        c["vt"][0, 2, 1, 5] = bad
        c["kt"][0, 2, 0, 7] = bad
        out = f64(_run(c))
        seen = out[0, 2]
        assert np.isfinite(out[0, [0, 1, 3]]).all()
        assert not np.isfinite(seen[2:, 5]).any(), "the row that sees the value shows it"
        assert np.isfinite(np.delete(seen[2:], 5, axis=1)).all(), "and only in the value's own dimension"
        c["q"] = c["q"][:, [0, 1, 3]].contiguous()
        c["kt"], c["vt"] = c["kt"][:, [0, 1, 3]].contiguous(), c["vt"][:, [0, 1, 3]].contiguous()
        c["n"], c["mask"] = 3, np.array([[0b001, 0b011, 0b101]], dtype=np.uint64)
        import torch
        _check(c, torch.from_numpy(out[:, [0, 1, 3]]), "others")


def test_mask_bits_past_n_and_skewed_scores():
    """Bits past n are ignored; scores far apart (one dominant key) and growing along the context."""
    masks = np.array([[0xFFFFFFFFFFFFFFF1, 0xF00000000000000F, 0x4, 0x8, 0x1F]], dtype=np.uint64)
    c = _case(1, 1, 8, 128, 5, 1024, [1000], seed=6, masks=masks)
    ramp = np.linspace(0.02, 6.0, 1000)[:, None]
    import torch
    c["k"][0, 0, :1000] *= torch.from_numpy(ramp).to(c["k"])
    _check(dict(c, mask=masks & np.uint64(0x1F)), _run(c), "skew")


def test_other_stream_and_repeat():
    import torch
    c = _case(3, 2, 4, 128, 9, 4096, [4000, 17, 2222], seed=8)
    first = _run(c)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        again = _run(c)
    third = _run(c, st.cuda_stream)
    assert torch.equal(first, again) and torch.equal(first, third)
    _check(c, first, "stream")


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes an entry's heads: the last head's last tokens are read in full."""
    import torch
    torch_cuda()
    Hkv, D, T_cap, T = 9, 128, 2_000_000, 1_999_990
    cfg = mkv.config(mkv.MKV_FP16, 1, Hkv, Hkv, D)
    k = torch.zeros((1, Hkv, T_cap, D), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    # one key that all the weight goes to, at the end of the last head
    q = torch.zeros((1, 1, Hkv, D), dtype=torch.float16, device="cuda")
    q[..., 0] = 40.0
    k[0, :, T - 1, 0] = 40.0
    v[0, :, T - 1] = torch.arange(Hkv, device="cuda", dtype=torch.float16)[:, None] + 1
    kt = torch.zeros((1, 1, Hkv, D), dtype=torch.float16, device="cuda")
    cache = caches.wrap_cache(cfg, torch.tensor([T], dtype=torch.int32, device="cuda"), k, v)
    ws, nws = caches.tree_workspace(cfg, T_cap, 1)
    out = torch.full_like(q, float("nan"))
    mask = torch.ones((1, 1), dtype=torch.int64, device="cuda")
    mkv.mkv_tree_attention(cfg, q.data_ptr(), cache.c, kt.data_ptr(), kt.data_ptr(), mask.data_ptr(), 1,
                           out.data_ptr(), ws.data_ptr(), nws)
    assert mkv.mkv_get_status() == 0
    np.testing.assert_allclose(f64(out[0, 0]), np.repeat(np.arange(1, Hkv + 1.0)[:, None], D, 1), rtol=1e-3)


# ------------------------------------------------------------------------------------------- commit
@pytest.mark.parametrize("D,Hkv,n", [(64, 1, 1), (128, 8, 16), (64, 3, 5), (128, 2, 70)])
def test_commit(D, Hkv, n):
    torch = torch_cuda()
    rng = np.random.default_rng(n)
    lens = [0, 7, 100, 33]
    B, T_cap = len(lens), 256
    c = _case(B, Hkv, 1, D, min(n, 64), T_cap, lens, seed=n)
    kt, vt = randn(rng, (B, n, Hkv, D), "fp16"), randn(rng, (B, n, Hkv, D), "fp16")
    paths = np.stack([rng.permutation(n) for _ in range(B)]).astype(np.int32)
    acc = [0, n, n // 2, 1]
    paths[2, acc[2]:] = 1 << 30                       # entries past the path are not read
    k0, v0 = c["k"].clone(), c["v"].clone()
    cfg = mkv.config(mkv.MKV_FP16, B, Hkv, Hkv, D)
    path = torch.from_numpy(paths).cuda()
    num = torch.tensor(acc, dtype=torch.int32, device="cuda")
    mkv.mkv_tree_commit(cfg, kt.data_ptr(), vt.data_ptr(), path.data_ptr(), num.data_ptr(), n, c["cache"].c)
    assert mkv.mkv_get_status() == 0
    for b in range(B):
        for i in range(acc[b]):
            k0[b, :, lens[b] + i] = kt[b, int(paths[b, i])]
            v0[b, :, lens[b] + i] = vt[b, int(paths[b, i])]
    assert torch.equal(c["k"], k0) and torch.equal(c["v"], v0)
    assert c["cache"].t["T_len"].tolist() == [t + a for t, a in zip(lens, acc)]


def test_commit_refuses_on_the_device_and_defaults():
    torch = torch_cuda()
    B, Hkv, D, n, T_cap = 5, 2, 64, 4, 16
    lens = [13, 12, 3, 3, 3]
    c = _case(B, Hkv, 1, D, n, T_cap, lens, seed=1)
    cfg = mkv.config(mkv.MKV_FP16, B, Hkv, Hkv, D)
    k0, v0 = c["k"].clone(), c["v"].clone()
    path = torch.tensor([[0, 1, 2, 3], [3, 2, 1, 0], [0, 4, 1, 2], [0, -1, 1, 2], [0, 1, 2, 3]], dtype=torch.int32,
                        device="cuda")
    num = torch.tensor([4, 4, 2, 2, 5], dtype=torch.int32, device="cuda")   # full, fits, bad index, bad index, too long
    mkv.mkv_tree_commit(cfg, c["kt"].data_ptr(), c["vt"].data_ptr(), path.data_ptr(), num.data_ptr(), n,
                        c["cache"].c)
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_CACHE_FULL
    assert c["cache"].t["T_len"].tolist() == [13, 16, 3, 3, 3]
    for i in range(4):
        k0[1, :, 12 + i], v0[1, :, 12 + i] = c["kt"][1, 3 - i], c["vt"][1, 3 - i]
    assert torch.equal(c["k"], k0) and torch.equal(c["v"], v0)
    # path and n_path NULL: a plain append of n tokens
    c["cache"].t["T_len"].fill_(2)
    mkv.mkv_tree_commit(cfg, c["kt"].data_ptr(), c["vt"].data_ptr(), 0, 0, n, c["cache"].c)
    assert mkv.mkv_get_status() == 0
    assert torch.equal(c["k"][:, :, 2:6], c["kt"].transpose(1, 2))
    assert c["cache"].t["T_len"].tolist() == [6] * B

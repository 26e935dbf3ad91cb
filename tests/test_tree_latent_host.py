"""Host-side refusals of the tree and latent entry points (no GPU needed)."""
import ctypes
import os

import pytest

import paper_2609_07966_gb300 as mkv

BIG = ctypes.c_size_t(1 << 40)
P = 1 << 20       # an aligned address that is never read: every call here is refused on the host


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mkv.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return mkv.lib()


def _cache(**kw):
    c = mkv.mkv_cache()
    c.T_cap, c.T_len, c.k, c.v = 256, P, P, P
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _tree(L, cfg=None, q=P, cache=None, kt=P, vt=P, mask=P, n=4, out=P, ws=P, nws=BIG):
    cfg = cfg or mkv.config(mkv.MKV_FP16, 2, 8, 2, 64)
    cache = cache or _cache()
    return L.mkv_tree_attention(ctypes.byref(cfg), q, ctypes.byref(cache), kt, vt, mask, n, out, ws, nws, None)


def test_tree_attention_refusals(L):
    inv, uns = mkv.MKV_ERR_INVALID_ARG, mkv.MKV_ERR_UNSUPPORTED
    for name in ("q", "kt", "vt", "mask", "out"):
        assert _tree(L, **{name: None}) == inv, name
    for name in ("q", "kt", "vt", "out"):
        assert _tree(L, **{name: P + 8}) == inv and "aligned" in mkv.mkv_last_error(), name
    assert _tree(L, cache=_cache(k=P + 2)) == inv and _tree(L, cache=_cache(T_len=None)) == inv
    assert _tree(L, cache=_cache(T_cap=0)) == inv
    assert _tree(L, n=0) == inv and _tree(L, n=-3) == inv
    assert _tree(L, n=65) == uns and "64" in mkv.mkv_last_error()
    assert _tree(L, cfg=mkv.config(mkv.MKV_H2O, 2, 8, 2, 64, h2o_heavy=4, h2o_recent=4)) == uns
    assert _tree(L, cfg=mkv.config(mkv.MKV_FP16, 2, 8, 2, 96)) == uns
    assert _tree(L, cfg=mkv.config(mkv.MKV_FP16, 2, 6, 2, 64)) == uns            # G = 3
    assert _tree(L, cache=_cache(T_cap=1 << 31)) == uns
    assert _tree(L, ws=None) == mkv.MKV_ERR_WORKSPACE
    assert _tree(L, nws=ctypes.c_size_t(64)) == mkv.MKV_ERR_WORKSPACE
    assert _tree(L, ws=P + 16) == inv
    with pytest.raises(mkv.MkvError):
        mkv.mkv_tree_workspace_size(mkv.config(mkv.MKV_FP16, 2, 8, 2, 64), 256, 65)
    small = mkv.mkv_tree_workspace_size(mkv.config(mkv.MKV_FP16, 1, 8, 2, 64), 256, 1)
    assert small <= mkv.mkv_tree_workspace_size(mkv.config(mkv.MKV_FP16, 1, 8, 2, 64), 256, 64)


def test_tree_commit_refusals(L):
    inv = mkv.MKV_ERR_INVALID_ARG
    cfg = mkv.config(mkv.MKV_FP16, 2, 8, 2, 64)

    def commit(cfg=cfg, kt=P, vt=P, n=3, cache=None):
        return L.mkv_tree_commit(ctypes.byref(cfg), kt, vt, None, None, n, ctypes.byref(cache or _cache()), None)
    assert commit(kt=None) == inv and commit(vt=None) == inv and commit(n=0) == inv
    assert commit(kt=P + 8) == inv and commit(cache=_cache(v=P + 4)) == inv
    assert commit(cfg=mkv.config(mkv.MKV_ROCKET, 1, 8, 2, 64, topk_pages=4, topq_dims=8, snap_window=8,
                                 snap_keep=64)) == mkv.MKV_ERR_UNSUPPORTED


def _lat(**kw):
    base = dict(dtype=mkv.MKV_F16, B=2, H=16)
    base.update(kw)
    return mkv.latent_config(base.pop("dtype"), base.pop("B"), base.pop("H"), **base)


def _lcache(**kw):
    c = mkv.mkv_latent_cache(256, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_latent_config_refusals(L):
    n = ctypes.c_size_t(0)

    def size(cfg, T=256, k=1):
        return L.mkv_latent_workspace_size(ctypes.byref(cfg) if cfg is not None else None, T, k, ctypes.byref(n))
    inv, uns = mkv.MKV_ERR_INVALID_ARG, mkv.MKV_ERR_UNSUPPORTED
    assert size(_lat()) == mkv.MKV_OK and n.value > 0
    assert size(None) == inv and size(_lat(dtype=2)) == inv and size(_lat(B=0)) == inv and size(_lat(H=0)) == inv
    assert size(_lat(softmax_scale=-1.0)) == inv and size(_lat(softmax_scale=float("inf"))) == inv
    for bad in (dict(rank=384), dict(rope_dim=32), dict(nope_dim=96), dict(v_dim=32), dict(H=257), dict(B=5000)):
        assert size(_lat(**bad)) == uns, bad
    assert size(_lat(), T=0) == inv and size(_lat(), k=0) == inv and size(_lat(), k=65) == uns
    assert size(_lat(), T=1 << 31) == uns
    assert size(_lat(B=4096, H=256), T=1 << 20, k=64) == uns and "tiles" in mkv.mkv_last_error()
    c = _lat()
    c.abi_version = 7
    assert size(c) == inv


def test_latent_call_refusals(L):
    inv, uns, wsp = mkv.MKV_ERR_INVALID_ARG, mkv.MKV_ERR_UNSUPPORTED, mkv.MKV_ERR_WORKSPACE
    cfg = _lat()
    by = ctypes.byref

    def attn(q=P, cache=None, new=P, mask=P, n=2, out=P, ws=P, nws=BIG):
        return L.mkv_latent_attention(by(cfg), q, by(cache or _lcache()), new, mask, n, out, ws, nws, None)
    assert attn(q=None) == inv and attn(out=None) == inv and attn(mask=None) == inv
    assert attn(q=P + 8) == inv and attn(new=P + 8) == inv and attn(out=P + 2) == inv and attn(ws=P + 64) == inv
    assert attn(cache=_lcache(rows=P + 8)) == inv and attn(cache=_lcache(rows=None)) == inv
    assert attn(n=0) == inv and attn(n=65) == uns
    assert attn(ws=None) == wsp and attn(nws=ctypes.c_size_t(8)) == wsp
    for f in (L.mkv_latent_absorb, L.mkv_latent_project):
        assert f(by(cfg), None, P, 1, P, None) == inv and f(by(cfg), P, None, 1, P, None) == inv
        assert f(by(cfg), P, P, 0, P, None) == inv and f(by(cfg), P, P, 1, P + 4, None) == inv

    def expand(T=256, w=P, kv=P, cache=None):
        return L.mkv_latent_expand(by(cfg), by(cache or _lcache()), w, T, kv, None)
    assert expand(T=0) == inv and expand(T=257) == inv and expand(w=None) == inv and expand(kv=P + 8) == inv
    assert expand(cache=_lcache(T_len=None)) == inv

    def prefill(q=P, kv=P, T=256, n=4, out=P, cfg=cfg):
        return L.mkv_latent_prefill(by(cfg), q, kv, T, by(_lcache()), None, n, out, None)
    assert prefill(q=None) == inv and prefill(kv=None) == inv and prefill(T=300) == inv and prefill(n=0) == inv
    assert prefill(out=P + 8) == inv and prefill(cfg=_lat(B=4096, H=17)) == uns
    assert L.mkv_latent_commit(by(cfg), None, None, None, 1, by(_lcache()), None) == inv
    assert L.mkv_latent_commit(by(cfg), P, None, None, 0, by(_lcache()), None) == inv
    assert L.mkv_latent_commit(by(cfg), P + 8, None, None, 1, by(_lcache()), None) == inv

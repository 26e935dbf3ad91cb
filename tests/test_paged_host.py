"""Host-side refusals of the rotary and paged entry points (no GPU needed)."""
import ctypes
import os

import pytest

import paper_2609_07966_gb300 as mkv
from paper_2609_07966_gb300 import caches

P = 1 << 20       # an aligned address that is never read: every call here is refused on the host
BIG = ctypes.c_size_t(1 << 40)
INV, UNS, WSP = mkv.MKV_ERR_INVALID_ARG, mkv.MKV_ERR_UNSUPPORTED, mkv.MKV_ERR_WORKSPACE
by = ctypes.byref


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mkv.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return mkv.lib()


def test_rope_config_refusals(L):
    def table(cfg, T=16, t=P):
        return L.mkv_rope_scaled_table(by(cfg) if cfg is not None else None, T, t, None)
    assert table(None) == INV
    for bad in (dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=130), dict(layout=2), dict(scaling=4), dict(theta=1.0),
                dict(theta=float("inf")), dict(theta=float("nan")), dict(magnitude=-1.0),
                dict(scaling=mkv.MKV_ROPE_LINEAR, factor=0.5),
                dict(scaling=mkv.MKV_ROPE_LINEAR, factor=float("inf")),
                dict(scaling=mkv.MKV_ROPE_BANDS, factor=2.0, context=0),
                dict(scaling=mkv.MKV_ROPE_BANDS, factor=2.0, context=8, low=4.0, high=4.0),
                dict(scaling=mkv.MKV_ROPE_RAMP, factor=2.0, context=8, low=0.0),
                dict(scaling=mkv.MKV_ROPE_RAMP, factor=2.0, context=8, high=float("inf"))):
        assert table(mkv.rope_config(128, **bad)) == INV, bad
    assert table(mkv.rope_config(3)) == INV and table(mkv.rope_config(0)) == INV
    assert table(mkv.rope_config(258)) == UNS
    good = mkv.rope_config(128)
    assert table(good, T=0) == INV and table(good, t=None) == INV and table(good, t=P + 4) == INV
    good.abi_version = 9
    assert table(good) == INV


def test_rope_apply_refusals(L):
    cfg = mkv.rope_config(64)

    def apply(dtype=mkv.MKV_F16, x=P, xs=0, pos=P, n=4, heads=8, t=P, T=16, out=2 * P, os=0):
        return L.mkv_rope_apply(by(cfg), dtype, x, xs, pos, n, heads, t, T, 0, out, os, None)
    for bad in (dict(dtype=2), dict(x=None), dict(pos=None), dict(out=None), dict(t=None), dict(n=0), dict(n=-1),
                dict(heads=0), dict(T=0), dict(x=P + 1), dict(out=P + 1), dict(pos=P + 2), dict(t=P + 4), dict(xs=511),
                dict(os=100), dict(xs=-512), dict(out=P, os=1024)):
        assert apply(**bad) == INV, bad
    assert apply(n=1 << 31) == UNS and apply(heads=65536) == UNS


def _cfg(**kw):
    base = dict(dtype=mkv.MKV_BF16, format=mkv.MKV_E4M3, B=2, Hq=8, Hkv=2, D=128, page_size=16)
    base.update(kw)
    return mkv.paged_config(**base)


def _cache(**kw):
    c = mkv.mkv_paged_cache(64, 8, P, P, P, P, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CONFIGS = [(dict(dtype=2), INV), (dict(format=2), INV), (dict(B=0), INV), (dict(Hq=0), INV), (dict(Hkv=0), INV),
               (dict(Hq=9), INV), (dict(softmax_scale=-1.0), INV), (dict(softmax_scale=float("nan")), INV),
               (dict(B=2049), UNS), (dict(Hq=66), UNS), (dict(D=96), UNS), (dict(page_size=8), UNS),
               (dict(page_size=48), UNS), (dict(page_size=256), UNS)]
BAD_CACHES = [(dict(num_pages=0), INV), (dict(max_pages=0), INV), (dict(num_pages=1 << 30), UNS),
              (dict(max_pages=1 << 28), UNS), (dict(k=P + 8), INV), (dict(v=P + 4), INV), (dict(k_scale=P + 2), INV),
              (dict(T_len=P + 1), INV)] + [(dict([(f, None)]), INV) for f in
                                          ("page_table", "T_len", "tickets", "k", "v", "k_scale", "v_scale")]


def test_append_refusals(L):
    rope = mkv.rope_config(128)
    base = dict(n=4, q=P, k=P, v=P, q_out=P)

    def append(cfg=None, cache=None, rope=rope, table=P, T=16, **kw):
        rows = mkv.paged_rows(**{**base, **kw})
        return L.mkv_paged_append(by(cfg or _cfg()), by(rope) if rope is not None else None, table, T, by(rows),
                                  by(cache or _cache()), None)
    for bad, status in BAD_CONFIGS:
        assert append(cfg=_cfg(**bad), rope=None) == status, bad
    for bad, status in BAD_CACHES:
        assert append(cache=_cache(**bad)) == status, bad
    for bad in (dict(n=0), dict(n=3), dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(k=P + 8),
                dict(q=P + 2), dict(start=P + 2), dict(pos=P + 1), dict(k_stride=252), dict(v_stride=128),
                dict(q_stride=1028), dict(q_out_stride=1032), dict(table=None), dict(table=P + 8), dict(T=0)):
        assert append(**bad) == INV, bad
    assert append(n=1 << 31, start=P) == UNS
    assert append(rope=mkv.rope_config(64)) == INV                     # another head's size
    assert append(rope=mkv.rope_config(128, rot_dim=40)) == UNS
    assert L.mkv_paged_append(by(_cfg()), None, None, 0, None, by(_cache()), None) == INV


def test_attention_refusals(L):
    def attend(cfg=None, cache=None, q=P, qs=0, start=None, n=4, most=2, out=P, os=0, ws=P, nws=BIG):
        return L.mkv_paged_attention(by(cfg or _cfg()), q, qs, start, n, most, by(cache or _cache()), out, os, ws, nws, None)
    for bad, status in BAD_CONFIGS:
        assert attend(cfg=_cfg(**bad)) == status, bad
    for bad, status in BAD_CACHES:
        assert attend(cache=_cache(**bad)) == status, bad
    for bad in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 2), dict(n=0), dict(n=3), dict(most=0),
                dict(most=5), dict(qs=1020), dict(os=512), dict(start=P + 2), dict(ws=P + 128)):
        assert attend(**bad) == INV, bad
    assert attend(ws=None) == WSP and attend(nws=ctypes.c_size_t(64)) == WSP
    assert attend(n=1 << 31, most=1) == UNS
    size = ctypes.c_size_t(0)
    assert L.mkv_paged_workspace_size(by(_cfg()), 4, 2, by(size)) == mkv.MKV_OK and size.value > 0
    assert attend(nws=ctypes.c_size_t(size.value - 1)) == WSP
    assert L.mkv_paged_workspace_size(by(_cfg()), 4, 2, None) == INV
    assert L.mkv_paged_workspace_size(by(_cfg()), 4, 5, by(size)) == INV


def test_wrapped_caches_are_checked():
    torch = pytest.importorskip("torch")
    cfg = _cfg()
    good = dict(page_table=torch.zeros(2, 8, dtype=torch.int32), T_len=torch.zeros(2, dtype=torch.int32),
                k=torch.zeros(64, 2, 16, 128).to(torch.float8_e4m3fn), v=torch.zeros(64, 2, 16, 128).to(torch.float8_e4m3fn),
                k_scale=torch.ones(64, 2), v_scale=torch.ones(64, 2))
    c = caches.wrap_paged_cache(cfg, **good)
    assert c.c.num_pages == 64 and c.c.max_pages == 8 and c.t["tickets"].shape == (2,)
    bad = dict(page_table=torch.zeros(1, 8, dtype=torch.int32), T_len=torch.zeros(2), k=good["k"].view(torch.int8),
               v=good["v"][:32], k_scale=torch.ones(64, 4), v_scale=torch.ones(64, 2).half())
    for name, value in bad.items():
        with pytest.raises(ValueError):
            caches.wrap_paged_cache(cfg, **{**good, name: value})
    for name in ("page_table", "k", "k_scale"):
        with pytest.raises(ValueError):
            caches.wrap_paged_cache(cfg, **{**good, name: good[name].transpose(0, 1)})
    with pytest.raises(ValueError):
        caches.wrap_paged_cache(cfg, **{**good, "k": good["k"][0]})
    with pytest.raises(ValueError):
        caches.wrap_paged_cache(cfg, **good, tickets=torch.zeros(1, dtype=torch.int32))


def test_attention_limits(L):
    def attend(cfg, cache, n=4, most=2, out=2 * P, qs=0, os=0):
        return L.mkv_paged_attention(by(cfg), P, qs, P, n, most, by(cache), out, os, P, ctypes.c_size_t(16), None)
    assert attend(_cfg(), _cache()) == WSP                # (all else is in order)
    assert attend(_cfg(), _cache(), out=P, os=2048) == INV
    assert attend(_cfg(), _cache(), out=P, qs=2048, os=2048) == WSP
    # query rows of a key head: 2^26
    assert attend(_cfg(), _cache(), n=1 << 25, most=(1 << 24)) == WSP
    assert attend(_cfg(), _cache(), n=1 << 25, most=(1 << 24) + 1) == UNS
    # tokens of all units: 2^36
    big = _cfg(B=64, Hq=32, Hkv=32, page_size=128)
    assert attend(big, _cache(max_pages=1 << 18)) == WSP
    assert attend(big, _cache(max_pages=(1 << 18) + 1)) == UNS


def test_workspace_grows_with_the_rows(L):
    """Never less for more rows: a workspace for the largest call serves the others; and it does not grow past 42 MB."""
    size = ctypes.c_size_t(0)
    for kw in (dict(), dict(D=64, Hq=32, Hkv=1), dict(B=1, Hq=3, Hkv=3)):
        last = 0
        for most in (1, 2, 4, 8, 9, 16, 32, 33, 64, 65, 128, 129, 1000, 4096, 100000):
            assert L.mkv_paged_workspace_size(by(_cfg(**kw)), 1 << 20, most, by(size)) == mkv.MKV_OK
            assert last <= size.value <= 42 * 10 ** 6, (kw, most)
            last = size.value

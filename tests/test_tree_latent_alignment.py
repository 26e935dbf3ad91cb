"""Host refusals of misaligned integer arrays (no GPU needed): the kernels read masks as 64-bit and lengths and paths as
32-bit words, which must lie on their own size."""
import ctypes
import os

import pytest

import paper_2609_07966_gb300 as mkv

BIG = ctypes.c_size_t(1 << 40)
P = 1 << 20       # an aligned address that is never read: every call here is refused on the host
INV = mkv.MKV_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mkv.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return mkv.lib()


def _refused(status, name):
    assert status == INV and name in mkv.mkv_last_error() and "aligned" in mkv.mkv_last_error(), mkv.mkv_last_error()


def _fp16(T_len=P):
    c = mkv.mkv_cache()
    c.T_cap, c.T_len, c.k, c.v = 256, T_len, P, P
    return ctypes.byref(c)


def _rows(T_len=P):
    return ctypes.byref(mkv.mkv_latent_cache(256, T_len, P))


# A call whose workspace is missing is refused after its arrays have been looked at; P + 4 is as far as a mask may lie
# from a word's boundary and still be an int32's.
def test_tree_calls(L):
    cfg = ctypes.byref(mkv.config(mkv.MKV_FP16, 2, 8, 2, 64))

    def attn(mask=P, T_len=P, ws=None):
        return L.mkv_tree_attention(cfg, P, _fp16(T_len), P, P, mask, 4, P, ws, BIG, None)
    assert attn() == mkv.MKV_ERR_WORKSPACE
    for off in (1, 2, 4):
        _refused(attn(mask=P + off), "mask")
    for off in (1, 2):
        _refused(attn(T_len=P + off), "T_len")

    def commit(path=None, n_path=None, T_len=P):
        return L.mkv_tree_commit(cfg, P, P, path, n_path, 3, _fp16(T_len), None)
    _refused(commit(path=P + 2), "path")
    _refused(commit(n_path=P + 1), "n_path")
    _refused(commit(T_len=P + 2), "T_len")


def test_latent_calls(L):
    cfg = ctypes.byref(mkv.latent_config(mkv.MKV_F16, 2, 16))

    def attn(mask=P, T_len=P, ws=None):
        return L.mkv_latent_attention(cfg, P, _rows(T_len), P, mask, 4, P, ws, BIG, None)
    assert attn() == mkv.MKV_ERR_WORKSPACE
    for off in (1, 2, 4):
        _refused(attn(mask=P + off), "mask")
    _refused(attn(T_len=P + 2), "T_len")
    # without drafted rows the mask is not read
    assert L.mkv_latent_attention(cfg, P, _rows(), None, P + 4, 4, P, None, BIG, None) == mkv.MKV_ERR_WORKSPACE
    _refused(L.mkv_latent_expand(cfg, _rows(P + 2), P, 256, P, None), "T_len")
    _refused(L.mkv_latent_prefill(cfg, P, P, 256, _rows(P + 2), None, 4, P, None), "T_len")
    _refused(L.mkv_latent_prefill(cfg, P, P, 256, _rows(), P + 2, 4, P, None), "q_len")
    _refused(L.mkv_latent_commit(cfg, P, P + 2, None, 3, _rows(), None), "path")
    _refused(L.mkv_latent_commit(cfg, P, None, P + 2, 3, _rows(), None), "n_path")
    _refused(L.mkv_latent_commit(cfg, P, None, None, 3, _rows(P + 1), None), "T_len")

"""Rows whose scores are all minus infinity: softmax has no value for them (NaN), unlike rows that see nothing (zeros)."""
import numpy as np
import pytest

from oracle import latent as L

import tree_latent_calls as calls
from gpu_util import torch_cuda
from latent_util import check_attention, f64, randn

pytestmark = pytest.mark.gpu

INF = float("inf")
MASKS = np.array([[0b000, 0b001, 0b101], [0b000, 0b001, 0b110]], dtype=np.uint64)


def _check(out, ref, mag, dtype, what):
    """NaN exactly where the definition has no value; the other rows within the formats' bounds."""
    got, none = f64(out), np.isnan(ref)
    np.testing.assert_array_equal(np.isnan(got), none, err_msg=what)
    live = ~none.any(axis=1)
    assert (none.all(axis=1) | live).all()
    if live.any():
        check_attention(out[np.flatnonzero(live)], ref[live], mag[live], dtype, what)


def _reference(*args):
    with np.errstate(invalid="ignore"):
        return L.attend_visible(*args)


@pytest.mark.parametrize("lens", [[0, 0], [1, 130], [700, 65]])
@pytest.mark.parametrize("T_cap", [720, 9000])
def test_tree(lens, T_cap):
    """Entry 0's keys are all minus infinity in a dim where every query is positive, entry 1's but one."""
    torch_cuda()
    rng = np.random.default_rng(1)
    B, n, Hkv, G, D = 2, 3, 2, 4, 64
    q, kt, vt = randn(rng, (B, n, Hkv * G, D), "fp16"), *(randn(rng, (B, n, Hkv, D), "fp16") for _ in range(2))
    k, v = (randn(rng, (B, Hkv, T_cap, D), "fp16") for _ in range(2))
    q[..., 3] = 1.0
    k[..., 3] = kt[..., 3] = -INF
    k[1, :, 64, 3] = 0.5
    kt[1, 2, :, 3] = 0.5
    out = calls.tree(q, k, v, lens, kt, vt, MASKS)
    for b, t in enumerate(lens):
        vis = np.repeat(L.tree_visible(MASKS[b], n, t), G, axis=0)
        for h in range(Hkv):
            keys, vals = (np.concatenate([f64(x[b, h, :t]), f64(y[b, :, h])]) for x, y in ((k, kt), (v, vt)))
            ref, mag = _reference(f64(q[b, :, h * G:(h + 1) * G]).reshape(n * G, D), keys, vals, vis, D ** -0.5)
            _check(out[b, :, h * G:(h + 1) * G].reshape(n * G, D), ref, mag, "fp16", f"b{b} h{h}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("H", [4, 32])
@pytest.mark.parametrize("lens", [[0, 0], [1, 130], [700, 65]])
@pytest.mark.parametrize("T_cap", [720, 9000])
def test_latent(dtype, H, lens, T_cap):
    torch_cuda()
    rng = np.random.default_rng(2)
    B, n, rank = 2, 3, 256
    q, new = randn(rng, (B, n, H, rank + 64), dtype), randn(rng, (B, n, rank + 64), dtype)
    rows = randn(rng, (B, T_cap, rank + 64), dtype)
    q[..., rank] = 1.0
    rows[..., rank] = new[..., rank] = -INF
    rows[1, 64, rank] = 0.5
    new[1, 2, rank] = 0.5
    out = calls.latent(dtype, q, rows, lens, new, MASKS)
    for b, t in enumerate(lens):
        keys = np.concatenate([f64(rows[b, :t]), f64(new[b])])
        vis = np.repeat(L.tree_visible(MASKS[b], n, t), H, axis=0)
        ref, mag = _reference(f64(q[b]).reshape(n * H, -1), keys, keys[:, :rank], vis, 192 ** -0.5)
        _check(out[b].reshape(n * H, rank), ref, mag, dtype, f"b{b}")


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_prefill(dtype):
    """Head 0's keys are all minus infinity; head 1's up to token 150; 60 queries lie before position 0."""
    import torch
    torch_cuda()
    rng = np.random.default_rng(3)
    B, n, H, T, lens = 2, 300, 3, 300, [300, 240]
    q, kv = randn(rng, (B, n, H, 128), dtype), randn(rng, (B, H, T, 128), dtype)
    rope = randn(rng, (B, T, 64), dtype)
    q[..., 5] = 1.0
    kv[:, 0, :, 5] = -INF
    kv[:, 1, :150, 5] = -INF
    out = calls.prefill(dtype, q, kv, rope, lens)
    assert torch.equal(out[1, :60], torch.zeros_like(out[1, :60]))
    for b, t in enumerate(lens):
        vis = L.causal_visible(n, n, t)
        for h in range(H):
            keys = np.concatenate([f64(kv[b, h, :t, :64]), f64(rope[b, :t])], 1)
            ref, mag = _reference(f64(q[b, :, h]), keys, f64(kv[b, h, :t, 64:]), vis, 128 ** -0.5)
            _check(out[b, :, h], ref, mag, dtype, f"b{b} h{h}")

"""Attention whose scores are far from zero: the weights depend on differences of scores alone."""
import numpy as np
import pytest

from oracle import latent as L

import tree_latent_calls as calls
from gpu_util import torch_cuda
from latent_util import check_attention, f64, randn

pytestmark = pytest.mark.gpu

# Every query is q in each of its rotated dims and zero elsewhere, every key k there, but for one key (`better`), so
# that all scores but one are the same number and the expected weights are 1 / count or 0 and 1.
SCORES = [("fp16", 60000.0, 60000.0, 60032.0), ("fp16", 60000.0, -60000.0, -59968.0),
          ("bf16", 2.0 ** 20, 2.0 ** 20, 1.5 * 2.0 ** 20)]


def _prefill(dtype, q0, k0, better):
    import torch
    rng = np.random.default_rng(5)
    B, n, H, T, lens, at = 2, 300, 2, 300, [300, 210], 170
    q = torch.zeros((B, n, H, 192), device="cuda")
    q[..., 128:] = q0
    kv = randn(rng, (B, H, T, 256), dtype)
    rope = torch.full((B, T, 64), k0, device="cuda")
    rope[1, at] = better
    q, rope = q.to(kv.dtype), rope.to(kv.dtype)
    out = calls.prefill(dtype, q, kv, rope, lens)
    for b, t in enumerate(lens):
        vis = L.causal_visible(n, n, t)
        for h in range(H):
            keys = np.concatenate([f64(kv[b, h, :t, :128]), f64(rope[b, :t])], 1)
            ref, mag = L.attend_visible(f64(q[b, :, h]), keys, f64(kv[b, h, :t, 128:]), vis, 192 ** -0.5)
            check_attention(out[b, :, h], ref, mag, dtype, f"b{b} h{h}")


@pytest.mark.parametrize("dtype,q0,k0,better", SCORES)
def test_prefill_large_scores(dtype, q0, k0, better):
    """Past 2^31 a score times the scale, unrounded, is hundreds away from the rounded maximum."""
    torch_cuda()
    _prefill(dtype, q0, k0, better)


# Negative scores near the end of the bf16 range's products: below -1e30.
FAR = [("bf16", 2.0 ** 60, -2.0 ** 50, -2.0 ** 49), ("bf16", 2.0 ** 60, 2.0 ** 50, 2.0 ** 51)]


@pytest.mark.parametrize("dtype,q0,k0,better", FAR)
def test_prefill_far_scores(dtype, q0, k0, better):
    torch_cuda()
    _prefill(dtype, q0, k0, better)


@pytest.mark.parametrize("dtype,q0,k0,better", SCORES + FAR)
@pytest.mark.parametrize("T_cap", [320, 9000])
def test_latent_far_scores(dtype, q0, k0, better, T_cap):
    import torch
    torch_cuda()
    rng = np.random.default_rng(6)
    B, n, H, lens, at, rank = 2, 2, 8, [300, 210], 170, 256
    q = torch.zeros((B, n, H, rank + 64), device="cuda")
    q[..., rank:] = q0
    rows = randn(rng, (B, T_cap, rank + 64), dtype)
    new = randn(rng, (B, n, rank + 64), dtype)
    rows[..., rank:] = k0
    new[..., rank:] = k0
    rows[1, at, rank:] = better
    q = q.to(rows.dtype)
    masks = np.array([[0b01, 0b11]] * B, dtype=np.uint64)
    out = calls.latent(dtype, q, rows, lens, new, masks)
    for b, t in enumerate(lens):
        keys = np.concatenate([f64(rows[b, :t]), f64(new[b])])
        vis = np.repeat(L.tree_visible(masks[b], n, t), H, axis=0)
        ref, mag = L.attend_visible(f64(q[b]).reshape(n * H, -1), keys, keys[:, :rank], vis, 192 ** -0.5)
        check_attention(out[b].reshape(n * H, rank), ref, mag, dtype, f"b{b}")

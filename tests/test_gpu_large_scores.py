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

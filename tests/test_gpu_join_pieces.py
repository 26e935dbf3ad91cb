"""A row's result does not depend on how its tokens were shared out: infinities and NaN, whatever the plan."""
import numpy as np
import pytest

from oracle import latent as L

import tree_latent_calls as calls
from gpu_util import torch_cuda
from latent_util import check_attention, f64, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T_cap", [704, 4000, 9000])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("where", ["cached", "drafted"])
def test_far_below_the_maximum(T_cap, bad, where):
    """A value that is not finite, of a token whose weight rounds to zero beside the others': its dim of every row that
    sees the token is not finite, be the tokens one CTA's, a cluster's or several runs' (by the capacity)."""
    torch_cuda()
    rng = np.random.default_rng(4)
    B, n, Hkv, G, D, T = 1, 3, 8, 4, 128, 700
    masks = np.array([[0b001, 0b011, 0b101]], dtype=np.uint64)
    q, k, v = randn(rng, (B, n, Hkv * G, D), "fp16"), *(randn(rng, (B, Hkv, T_cap, D), "fp16") for _ in range(2))
    kt, vt = (randn(rng, (B, n, Hkv, D), "fp16") for _ in range(2))
    q[..., 0] = 30.0                       # scores 114 apart from zero either way (log2), 2^-228 between them
    k[..., 0], kt[..., 0] = 30.0, 30.0
    if where == "cached":
        k[0, :, :300, 0] = -30.0
        v[0, 2, 100, 7] = bad
        hit = [0, 1, 2]
    else:
        kt[0, 1, :, 0] = -30.0
        vt[0, 1, 2, 7] = bad
        hit = [1]
    out = f64(calls.tree(q, k, v, [T], kt, vt, masks))
    expect = np.ones(out.shape, bool)
    for i in hit:
        expect[0, i, 2 * G:3 * G, 7] = False
    np.testing.assert_array_equal(np.isfinite(out), expect)
    vis = np.repeat(L.tree_visible(masks[0], n, T), G, axis=0)
    for h in range(Hkv):
        keys, vals = (np.concatenate([f64(x[0, h, :T]), f64(y[0, :, h])]) for x, y in ((k, kt), (v, vt)))
        vals[~np.isfinite(vals)] = 0.0     # (dims beside the value's own)
        ref, mag = L.attend_visible(f64(q[0, :, h * G:(h + 1) * G]).reshape(n * G, D), keys, vals, vis, D ** -0.5)
        got = out[0, :, h * G:(h + 1) * G].reshape(n * G, D)
        ok = np.isfinite(got)
        import torch
        check_attention(torch.from_numpy(np.where(ok, got, 0.0)), np.where(ok, ref, 0.0), mag, "fp16", f"h{h}")

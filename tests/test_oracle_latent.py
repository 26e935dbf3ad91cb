"""The latent / tree oracle against brute force, the dense oracle and the identity of its two forms (CPU)."""
import numpy as np
import pytest

from oracle import attention, latent


def test_full_visibility_is_plain_attention():
    rng = np.random.default_rng(0)
    q, K, V = rng.standard_normal((5, 8)), rng.standard_normal((11, 8)), rng.standard_normal((11, 6))
    out, mag = latent.attend_visible(q, K, V, np.ones((5, 11), bool), 0.3)
    ref, *_ = attention.attend(q, K, V, 0.3)
    np.testing.assert_allclose(out, ref, rtol=1e-12, atol=1e-14)
    assert (mag >= np.abs(out) - 1e-15).all()


def test_invisible_keys_do_not_matter_and_empty_rows_are_zero():
    rng = np.random.default_rng(1)
    q, K, V = rng.standard_normal((3, 4)), rng.standard_normal((6, 4)), rng.standard_normal((6, 4))
    vis = np.zeros((3, 6), bool)
    vis[0, [1, 4]] = vis[2, 3] = True
    K2, V2 = K.copy(), V.copy()
    K2[[0, 2, 5]], V2[[0, 2, 5]] = np.nan, np.inf
    a, _ = latent.attend_visible(q, K, V, vis, 1.0)
    b, _ = latent.attend_visible(q, K2, V2, vis, 1.0)
    np.testing.assert_array_equal(a, b)
    assert (a[1] == 0).all()
    np.testing.assert_allclose(a[2], V[3], rtol=1e-15)
    s = np.exp(q[0] @ K[1]), np.exp(q[0] @ K[4])
    np.testing.assert_allclose(a[0], (s[0] * V[1] + s[1] * V[4]) / (s[0] + s[1]), rtol=1e-12)


def test_visibility_patterns():
    vis = latent.tree_visible([0b001, 0b011, 0b101], 3, 2)
    assert vis.astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 1, 0, 1]]
    assert latent.causal_visible(2, 3, 4).astype(int).tolist() == [[1, 1, 1, 0], [1, 1, 1, 1], [0, 0, 0, 0]]
    assert latent.causal_visible(3, 3, 1).astype(int).tolist() == [[0], [0], [1]]


@pytest.mark.parametrize("dims", [(16, 8, 4, 12, 6), (24, 4, 8, 4, 10)])
def test_absorbed_and_expanded_forms_agree(dims):
    r, rope, H, nope, dv = dims
    rng = np.random.default_rng(2)
    T, n = 9, 3
    c = rng.standard_normal((T, r + rope))
    w = rng.standard_normal((H, nope + dv, r))
    q = rng.standard_normal((n, H, nope + rope))
    vis = latent.causal_visible(n, n, T)
    kv = latent.expand(c[:, :r], w)
    qa = latent.absorb(q, w[:, :nope], nope)
    for h in range(H):
        K = np.concatenate([kv[h, :, :nope], c[:, r:]], 1)
        full, _ = latent.attend_visible(q[:, h], K, kv[h, :, nope:], vis, 0.2)
        lat, _ = latent.attend_visible(qa[:, h], c, c[:, :r], vis, 0.2)
        np.testing.assert_allclose(latent.project(lat[:, None], w[h:h + 1, nope:])[:, 0], full, rtol=1e-10, atol=1e-12)

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


def _masks(B, n):
    """Token 2 is seen by itself alone, the others by their chain 0, 1, 3, 4, .."""
    m = []
    for i in range(n):
        m.append(0b100 if i == 2 else sum(1 << j for j in range(i + 1) if j != 2))
    return np.array([m] * B, dtype=np.uint64)


# (entries, key heads, group, drafted, capacity, lengths): many short units of unequal lengths, a CTA's run holding whole
# units and parts of others; few long ones, shared by many runs; several row blocks side by side
RUNS = [(90, 1, 2, 4, 512, [(37 * b * b) % 500 for b in range(90)]), (45, 2, 8, 3, 512, [(61 * b) % 400 for b in range(45)]),
        (2, 2, 4, 4, 8200, [8190, 5001]), (1, 2, 8, 20, 20010, [20000])]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("B,Hkv,G,n,T_cap,lens", RUNS)
def test_tree_runs_unseen_tokens_do_not_leak(D, bad, B, Hkv, G, n, T_cap, lens):
    """Every third entry's token 2 holds a value that is not finite: it reaches the rows that see it, in its dim, and
    neither the other rows nor the units that the same CTA works on next."""
    import torch
    torch_cuda()
    rng = np.random.default_rng(D + n)
    q, k, v = randn(rng, (B, n, Hkv * G, D), "fp16"), *(randn(rng, (B, Hkv, T_cap, D), "fp16") for _ in range(2))
    kt, vt = (randn(rng, (B, n, Hkv, D), "fp16") for _ in range(2))
    masks, hit = _masks(B, n), list(range(0, B, 3))
    kept = vt.clone()
    for b in hit:
        vt[b, 2, Hkv - 1, 5] = bad
    out = calls.tree(q, k, v, lens, kt, vt, masks)
    expect = np.ones(out.shape, bool)
    for b in hit:
        expect[b, 2, (Hkv - 1) * G:, 5] = False
    np.testing.assert_array_equal(np.isfinite(f64(out)), expect)
    assert torch.equal(out[torch.from_numpy(~expect)].isnan().any(), torch.tensor(np.isnan(bad), device="cuda"))
    for b in range(B) if B < 10 else range(0, B, 7):
        t, vis = lens[b], np.repeat(L.tree_visible(masks[b], n, lens[b]), G, axis=0)
        for h in range(Hkv):
            keys, vals = (np.concatenate([f64(x[b, h, :t]), f64(y[b, :, h])]) for x, y in ((k, kt), (v, kept)))
            ref, mag = L.attend_visible(f64(q[b, :, h * G:(h + 1) * G]).reshape(n * G, D), keys, vals, vis, D ** -0.5)
            ok = expect[b, :, h * G:(h + 1) * G].reshape(n * G, D)
            got = out[b, :, h * G:(h + 1) * G].reshape(n * G, D).cpu()
            check_attention(got.masked_fill(torch.from_numpy(~ok), 0.0), np.where(ok, ref, 0.0), mag, "fp16", f"b{b} h{h}")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,B,H,rank,n,T_cap,lens", [
    ("bf16", 90, 8, 256, 3, 320, [(29 * b * b) % 300 for b in range(90)]), ("fp16", 2, 16, 512, 4, 8200, [8190, 5001]),
    ("bf16", 1, 32, 512, 6, 20010, [20000]), ("bf16", 2, 128, 256, 20, 80, [70, 3])])
def test_latent_runs_unseen_tokens_do_not_leak(dtype, bad, B, H, rank, n, T_cap, lens):
    """As above; a latent row's value is part of its key too, so all dims of the rows that see it are lost.  The last
    shape has forty row blocks an entry, worked on one after another."""
    import torch
    torch_cuda()
    rng = np.random.default_rng(B + H)
    q, new = randn(rng, (B, n, H, rank + 64), dtype), randn(rng, (B, n, rank + 64), dtype)
    rows = randn(rng, (B, T_cap, rank + 64), dtype)
    masks, hit = _masks(B, n), list(range(0, B, 3))
    for b in hit:
        new[b, 2, 9] = bad
    out = calls.latent(dtype, q, rows, lens, new, masks)
    expect = np.ones(out.shape, bool)
    for b in hit:
        expect[b, 2] = False
    got = f64(out)
    assert np.isfinite(got[expect]).all()
    for b in hit:
        assert not np.isfinite(got[b, 2, :, 9]).any()
    for b in range(B) if B < 10 else range(0, B, 7):
        t, keep = lens[b], [i for i in range(n) if i != 2]
        keys = np.concatenate([f64(rows[b, :t]), f64(new[b, keep])])
        vis = L.tree_visible(masks[b], n, t)[keep][:, list(range(t)) + [t + j for j in keep]]
        ref, mag = L.attend_visible(f64(q[b, keep]).reshape(len(keep) * H, -1), keys, keys[:, :rank],
                                    np.repeat(vis, H, axis=0), 192 ** -0.5)
        check_attention(out[b, keep].reshape(len(keep) * H, rank), ref, mag, dtype, f"b{b}")

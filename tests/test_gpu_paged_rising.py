"""Attention over 8-bit pages where the running maxima rise again and again, so that sums and outputs are scaled down in tile
after tile: scores that grow along the sequence, value scales that do, and scores that grow as value scales fall.

Errors, in the terms of latent_util.py, with S the largest scale sum |q k| of what a row sees, in nats: the accumulation of a
score is off by 2^-22 S per 16 products; its factor has three roundings (2^-24 S each), the maximum and the shift that are
taken off one each, of numbers below S + 45 (64 in log2), and the difference one: together less than 2 x 2^-22 (S + 45).  A
weight below fp16's normal range is off by 2^-25, which is 2^-31 of the largest weight that a row could have (2^6 or more,
see paged_util.py), so 2^-31 of max_t p_t vs_t times the largest code, a token.  Joined sums add a few 2^-22, less than 2^-18.
"""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import paged as P

from gpu_util import torch_cuda
from latent_util import TINY, U, f64
from paged_util import device, seeded
from test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu

LOG2E = np.log2(np.e)
LEVEL = 64.0                        # of the keys' codes along a head's direction


def attend(q, k, ks, v, vs, visible, scale):
    """One key head: q [R, D], codes k, v [T, D] with their scales [T], visible [R, T].  Output, mean |v|, S and the largest
    p vs of each row."""
    s = scale * (q @ k.T) * ks
    size = np.where(visible, scale * (np.abs(q) @ np.abs(k).T) * ks, 0.0).max(axis=1)
    s = np.where(visible, s, -np.inf)
    p = np.exp(s - s.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    w = p * vs
    return w @ v, w @ np.abs(v), size[:, None], w.max(axis=1)[:, None]


class Rising(Case):
    """Every row's score of a token is about level(token) in log2, which rises by 9 to 12 from some tiles to the next (all of
    them with `often` 1); value scales are 2^-level (kind "apart"), 2^(level - the last one) with scores that stay
    ("values"), or about 1."""

    def __init__(self, dtype, fmt, D, page, lens, new, kind, often, **kw):
        super().__init__(dtype, fmt, 8, 2, D, page, lens, new, **kw)
        torch = torch_cuda()
        hc, Hkv, G = self.hc, self.cfg.Hkv, self.cfg.Hq // self.cfg.Hkv
        rng = seeded("rising", dtype, fmt, D, page, tuple(lens), tuple(new), kind, often)
        u = np.where(rng.random((Hkv, D)) < 0.5, -1.0, 1.0)
        per = lambda level: level / (D ** -0.5 * LOG2E * LEVEL * D)         # the key scale that gives this level
        for b in range(self.cfg.B):
            for h in range(Hkv):
                tiles = hc.table.shape[1] * page // 128 + 1
                rise = np.where(rng.random(tiles) < often, rng.uniform(9.0, 12.0, tiles), 0.0)
                level = np.minimum(4.0 + np.cumsum(rise) - rise[0], 110.0)
                for p in range(hc.table.shape[1]):
                    pid, at = hc.table[b, p], level[p * page // 128] + rng.uniform(-1.0, 1.0)
                    x = LEVEL * u[h] + 6.0 * rng.standard_normal((page, D))
                    hc.k[pid, h] = P.encode(x.astype(np.float32), fmt)
                    hc.ks[pid, h] = per(4.0 if kind == "values" else at)
                    if kind != "scores":
                        hc.vs[pid, h] *= 2.0 ** (at - level[-1] if kind == "values" else -at)
        for name, x in (("k", hc.k), ("k_scale", hc.ks), ("v_scale", hc.vs)):
            t = hc.cache.t[name]
            t.view(torch.uint8 if name == "k" and fmt == "e4m3" else t.dtype).copy_(device(x))
        q = np.repeat(u, G, axis=0)[None] * (1.0 + 0.1 * rng.standard_normal((self.q.shape[0], 8, D)))
        self.q.copy_(device(q.astype(np.float32)))

    def check(self):
        torch = torch_cuda()
        torch.cuda.synchronize()
        assert mkv.mkv_get_status() == 0
        hc, page, D = self.hc, self.hc.page, self.cfg.D
        G, q, got = self.cfg.Hq // self.cfg.Hkv, f64(self.q), f64(self.out)
        for b, t in enumerate(hc.lens):
            r0, r1 = self.starts[b], self.starts[b + 1]
            m, ids = r1 - r0, hc.table[b, :-(-t // page)]
            vis = np.repeat(np.arange(t)[None, :] <= (t - m + np.arange(m))[:, None], G, axis=0)
            for h in range(self.cfg.Hkv if m else 0):
                k, v = (P.decode(x[ids, h], self.fmt).reshape(-1, D)[:t] for x in (hc.k, hc.v))
                ks, vs = (np.repeat(x[ids, h].astype(np.float64), page)[:t] for x in (hc.ks, hc.vs))
                mine = lambda x: x[r0:r1, h * G:(h + 1) * G].reshape(m * G, D)
                ref, mag, size, most = attend(mine(q), k, ks, v, vs, vis, D ** -0.5)
                d = 2.0 ** -22 * (D / 16 + 2) * (size + 45)
                tol = (U["fp16"] + 2 * d + 2.0 ** -18) * mag + U[self.dtype] * np.abs(ref) \
                    + t * 2.0 ** -31 * np.abs(v).max() * most + TINY[self.dtype]
                bad = ~(np.abs(mine(got) - ref) <= tol)
                assert not bad.any(), f"b{b} h{h}: {int(bad.sum())} of {bad.size} off, worst of tolerances " \
                                      f"{np.nanmax(np.abs(mine(got) - ref) / tol):.2f}, first {np.argwhere(bad)[0].tolist()}"

    @property
    def fmt(self):
        return self.hc.fmt


KINDS = [("fp16", "e4m3", "scores"), ("bf16", "int8", "scores"), ("fp16", "int8", "scores"), ("bf16", "e4m3", "scores"),
         ("bf16", "int8", "values"), ("bf16", "e4m3", "apart")]


def run_and_check(c):
    """Right, and bit for bit the same however the warps happen to run."""
    torch = torch_cuda()
    want = c.run().clone()
    c.check()
    for _ in range(8):
        c.out[:c.n].fill_(0)
        c.run()
        assert torch.equal(c.out, want)


# most new tokens of an entry, times 4 heads a group: 8, 32, 64, 120 and 280 query rows a key head
@pytest.mark.parametrize("most", [2, 8, 16, 30, 70])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype,fmt,kind", KINDS)
def test_every_tile(most, D, page, dtype, fmt, kind):
    """Units of up to eight tiles, each above the one before."""
    run_and_check(Rising(dtype, fmt, D, page, [1000, 517, 130], [most, max(1, most // 2), most], kind, 1.0))


@pytest.mark.parametrize("most", [2, 8, 16, 30, 70])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype,fmt,kind", KINDS[:2] + KINDS[4:])
def test_some_tiles_of_long_units(most, D, page, dtype, fmt, kind):
    """Units that several CTAs share, with maxima of their own."""
    run_and_check(Rising(dtype, fmt, D, page, [2900, 300, 1611], [most, 1, most], kind, 0.35))


@pytest.mark.parametrize("dtype,fmt", [("fp16", "e4m3"), ("bf16", "int8")])
def test_a_prompt(dtype, fmt):
    """Many blocks of rows over tiles that all rise."""
    run_and_check(Rising(dtype, fmt, 128, 64, [1000, 700], [1000, 641], "scores", 1.0))


@pytest.mark.parametrize("D", [64, 128])
def test_many_units(D):
    """Every SM at work, several CTAs after one another."""
    run_and_check(Rising("fp16", "e4m3", D, 32, [900 - 7 * b for b in range(30)], [300 - 5 * b for b in range(30)], "scores", 1.0))

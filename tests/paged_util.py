"""Helpers of the rotary and 8-bit paged cache tests: caches made on the host, and what tolerances follow from.

Attention: weights are rounded to fp16 (2^-11 of mean |v|), what lies below their normal range by 2^-31 of the largest |v|
a token, the output to its type; a score is off by less than SCORE (tests/latent_util.py) for inputs of this size.
"""
import numpy as np

import paper_2609_07966_gb300 as mkv
from oracle import paged as P
from oracle.latent import attend_visible
from paper_2609_07966_gb300 import caches

from latent_util import SCORE, TINY, U, f64, torch_dtype

KINDS = {"fp16": mkv.MKV_F16, "bf16": mkv.MKV_BF16}
FORMATS = {"e4m3": mkv.MKV_E4M3, "int8": mkv.MKV_I8}
LAYOUTS = {"half": mkv.MKV_ROPE_HALF, "pairs": mkv.MKV_ROPE_PAIRS}


def seeded(*key):
    """A generator from plain values alone (hash() of a text changes from process to process)."""
    import zlib
    return np.random.default_rng(zlib.crc32(repr(key).encode()))


def device(a, dtype=None, dev="cuda"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t.to(dtype) if dtype is not None else t).to(dev)


class HostCache:
    """Random pages in numpy, and the same on the device."""

    def __init__(self, rng, cfg, fmt, lens, max_pages, spare=3, pow2=False, wild=0):
        import torch
        B, Hkv, D, page = cfg.B, cfg.Hkv, cfg.D, cfg.page_size
        self.cfg, self.fmt, self.page = cfg, fmt, page
        num = B * max_pages + spare
        self.table = rng.permutation(num)[:B * max_pages].reshape(B, max_pages).astype(np.int32)
        self.lens = np.array(lens, dtype=np.int32)
        shape = (num, Hkv, page, D)
        x = rng.standard_normal((2,) + shape).astype(np.float32)
        self.k, self.v = (P.encode(y * (32 if fmt == "int8" else 112), fmt) for y in x)
        base = 2.0 ** -5 if fmt == "int8" else 2.0 ** -7
        e = rng.integers(-1 - wild, 2 + wild, (2, num, Hkv)).astype(np.float64)
        f = np.ones_like(e) if pow2 else rng.uniform(0.75, 1.25, e.shape)
        self.ks, self.vs = (base * f * 2.0 ** e).astype(np.float32)
        if wild:                              # (keys of usual size: their scores are held to SCORE)
            self.ks = (base * f[0]).astype(np.float32)
        t8 = caches.code_dtype(cfg)
        self.cache = caches.wrap_paged_cache(cfg, device(self.table), device(self.lens), device(self.k).view(t8),
                                             device(self.v).view(t8), device(self.ks), device(self.vs))
        assert torch.cuda.is_available()

    def tokens(self, b, h, n):
        """Entry b's first n keys and values of head h, fp64."""
        ids = self.table[b, :-(-n // self.page)]
        out = []
        for c, s in ((self.k, self.ks), (self.v, self.vs)):
            x = P.decode(c[ids, h], self.fmt) * s[ids, h].astype(np.float64)[:, None, None]
            out.append(x.reshape(-1, x.shape[-1])[:n])
        return out

    def device_codes(self, name):
        import torch
        t = self.cache.t[name]
        return t.view(torch.uint8 if self.fmt == "e4m3" else torch.int8).cpu().numpy()


def check_attention(hc, q, starts, out, dtype, scale=None, what="", seen=None, entries=None):
    """out [n][Hq][D] against the oracle; starts: rows of each entry; seen(b, t): bool mask of tokens that exist."""
    cfg = hc.cfg
    G = cfg.Hq // cfg.Hkv
    scale = cfg.D ** -0.5 if scale is None else scale
    q, got = f64(q), f64(out)
    for b in range(cfg.B) if entries is None else entries:
        r0, r1 = starts[b], starts[b + 1]
        m, t = r1 - r0, int(hc.lens[b])
        if m == 0:
            continue
        vis = np.arange(t)[None, :] <= (t - m + np.arange(m))[:, None]
        if seen is not None:
            vis = vis & seen(b, t)[None, :]
        for h in range(cfg.Hkv):
            K, V = hc.tokens(b, h, t)
            rows = q[r0:r1, h * G:(h + 1) * G].reshape(m * G, -1)
            ref, mag = attend_visible(rows, K, V, np.repeat(vis, G, axis=0), scale)
            g = got[r0:r1, h * G:(h + 1) * G].reshape(m * G, -1)
            vmax = np.abs(V).max() if t else 0.0
            tol = (U["fp16"] + 2 * SCORE) * mag + U[dtype] * np.abs(ref) + t * 2.0 ** -31 * vmax + TINY[dtype]
            bad = ~(np.abs(g - ref) <= tol)
            assert not bad.any(), f"{what} b{b} h{h}: {int(bad.sum())} of {bad.size} off, worst " \
                                  f"{np.abs(g - ref).max():.3e}, first at {np.argwhere(bad)[0].tolist()}"

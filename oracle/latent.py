"""O9: attention under an arbitrary visibility pattern, and the two forms of latent attention (fp64).

A drafted token sees the cached tokens and its own branch of the tree; a prompt's query sees the tokens up
to its own.  Both are softmax attention over a row's visible set; a row that sees nothing gives zeros.

Latent attention stores c_t = [latent | rotated key] a token; head h's key is [W_uk c_t[:r] | c_t[r:]] and its
value W_uv c_t[:r].  Because both are linear, W_uk can move to the query and W_uv behind the sum:
    q_nope . (W_uk c) = (W_uk^T q_nope) . c,     sum_t p_t W_uv c_t = W_uv sum_t p_t c_t.
"""
from __future__ import annotations

import numpy as np


def attend_visible(q, K, V, visible, scale):
    """q [R, dk], K [n, dk], V [n, dv], visible bool [R, n] -> (out [R, dv], mean |v| under the weights [R, dv]).

    Each row is computed over its visible keys alone, so what it does not see cannot reach it.
    """
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    out = np.zeros((q.shape[0], V.shape[1]))
    mag = np.zeros_like(out)
    for i in range(q.shape[0]):
        idx = np.flatnonzero(visible[i])
        if idx.size == 0:
            continue
        s = scale * (K[idx] @ q[i])
        e = np.exp(s - s.max())
        p = e / e.sum()
        out[i] = p @ V[idx]
        mag[i] = p @ np.abs(V[idx])
    return out, mag


def tree_visible(mask, n, T):
    """Visibility of n drafted tokens over T cached ones and each other: bits of mask [n] (Python ints or uint64)."""
    vis = np.zeros((n, T + n), dtype=bool)
    vis[:, :T] = True
    for i in range(n):
        for j in range(n):
            vis[i, T + j] = (int(mask[i]) >> j) & 1
    return vis


def causal_visible(q_len, n, T):
    """Query i < q_len is at position T - q_len + i; queries past q_len see nothing."""
    vis = np.zeros((n, T), dtype=bool)
    for i in range(min(n, q_len)):
        vis[i, :max(0, T - q_len + i + 1)] = True
    return vis


def absorb(q, w_uk, nope):
    """q [R, H, nope + rope], w_uk [H, nope, r] -> [R, H, r + rope]."""
    q, w_uk = np.asarray(q, dtype=np.float64), np.asarray(w_uk, dtype=np.float64)
    return np.concatenate([np.einsum("ihd,hdr->ihr", q[..., :nope], w_uk), q[..., nope:]], -1)


def project(o, w_uv):
    """o [R, H, r], w_uv [H, dv, r] -> [R, H, dv]."""
    return np.einsum("ihr,hdr->ihd", np.asarray(o, dtype=np.float64), np.asarray(w_uv, dtype=np.float64))


def expand(c, w_kv):
    """c [T, r], w_kv [H, d, r] -> [H, T, d]."""
    return np.einsum("tr,hdr->htd", np.asarray(c, dtype=np.float64), np.asarray(w_kv, dtype=np.float64))

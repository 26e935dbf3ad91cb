"""Speculative decoding with a latent cache, end to end on one layer.

A toy language model (random weights, one latent-attention layer) reads a prompt and then decodes with a draft: a cheap
guesser proposes a small tree of tokens behind the last one, a single pass attends with all of them, and the longest
branch that the model itself would have chosen is accepted.  It uses, in the order a server does,

    mkv_latent_commit     the prompt's rows, then every step's accepted path, join the cache
    mkv_latent_expand     the prompt's keys and values, once
    mkv_latent_prefill    the prompt's attention (expanded form)
    mkv_latent_absorb     a step's queries carried into the latent space
    mkv_latent_attention  the tree's attention over the cache and itself (absorbed form)
    mkv_latent_project    its outputs carried out again

and decodes the same prompt one token at a time beside it.  Run: python examples/speculative_decode.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2609_07966_gb300 as mkv  # noqa: E402
from paper_2609_07966_gb300 import caches  # noqa: E402

# A drafted token's parent in the tree; token 0 is the last accepted one, the others are guesses.
PARENT = [-1, 0, 0, 1, 1, 2, 3, 3]
DEPTH = [0, 1, 1, 2, 2, 2, 3, 3]
RANK = [0, 0, 1, 0, 1, 0, 0, 1]            # which of its parent's guesses it is


def tree_mask(parent):
    """Bits of the tokens that each token sees: itself and its ancestors."""
    m = []
    for j, p in enumerate(parent):
        m.append((m[p] if p >= 0 else 0) | 1 << j)
    return m


class Model:
    """tokens -> logits through x + W_o attention(x), with a latent cache of one row a token."""

    def __init__(self, B, capacity, seed=0, vocab=512, d=256, H=8, rank=256, nope=64, v=64, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.B, self.H, self.rank, self.nope, self.rope, self.v, self.dev = B, H, rank, nope, 64, v, device
        w = lambda *s, k: (torch.randn(s, generator=g, device=device) * k ** -0.5).half()      # noqa: E731
        self.embed = w(vocab, d, k=1)
        self.w_q, self.w_row = w(d, H * (nope + 64), k=d), w(d, rank + 64, k=d)
        self.w_kv = w(H, nope + v, rank, k=rank)
        self.w_o, self.head = w(H * v, d, k=H * v), w(d, vocab, k=d)
        self.cfg = mkv.latent_config(mkv.MKV_F16, B, H, rank=rank, nope_dim=nope, v_dim=v)
        self.cache = caches.alloc_latent_cache(self.cfg, capacity, device=device)
        self.ws, self.ws_bytes = caches.latent_workspace(self.cfg, capacity, len(PARENT), device=device)
        self.freq = 10000.0 ** (-torch.arange(32, device=device) / 32)

    def _rotate(self, x, pos):
        """Rotary embedding of the last 64 values (rotate-half) at positions pos."""
        a = pos.float()[..., None] * self.freq
        while a.dim() < x.dim():
            a = a.unsqueeze(-2)
        c, s = torch.cos(a), torch.sin(a)
        r = x[..., -64:].float()
        r = torch.cat([r[..., :32] * c - r[..., 32:] * s, r[..., 32:] * c + r[..., :32] * s], -1)
        return torch.cat([x[..., :-64], r.to(x.dtype)], -1).contiguous()

    def _inputs(self, tokens, pos):
        """tokens, pos [B][n] -> embeddings, rotated queries [B][n][H][..] and cache rows [B][n][rank + 64]."""
        x = self.embed[tokens]
        q = self._rotate((x @ self.w_q).reshape(*tokens.shape, self.H, -1), pos)
        return x, q, self._rotate(x @ self.w_row, pos)

    def _logits(self, x, attended):
        return (x + attended.reshape(*x.shape[:-1], -1) @ self.w_o) @ self.head

    def guess(self, tokens, k):
        """The draft: the k best next tokens by the embedding alone."""
        return (self.embed[tokens] @ self.head).float().topk(k, -1).indices

    def prefill(self, tokens):
        """Reads a prompt [B][T] into the cache; logits behind its last token."""
        B, T = tokens.shape
        pos = torch.arange(T, device=self.dev).expand(B, T)
        x, q, rows = self._inputs(tokens, pos)
        mkv.mkv_latent_commit(self.cfg, rows.data_ptr(), 0, 0, T, self.cache.c)
        kv = torch.empty(B, self.H, T, self.nope + self.v, dtype=torch.float16, device=self.dev)
        mkv.mkv_latent_expand(self.cfg, self.cache.c, self.w_kv.data_ptr(), T, kv.data_ptr())
        out = torch.empty(B, T, self.H, self.v, dtype=torch.float16, device=self.dev)
        mkv.mkv_latent_prefill(self.cfg, q.data_ptr(), kv.data_ptr(), T, self.cache.c, 0, T, out.data_ptr())
        return self._logits(x[:, -1], out[:, -1])

    def attend(self, tokens, pos, mask):
        """Logits [B][n][vocab] behind drafted tokens [B][n], and their cache rows (not yet committed)."""
        B, n = tokens.shape
        x, q, rows = self._inputs(tokens, pos)
        qa = torch.empty(B, n, self.H, self.rank + 64, dtype=torch.float16, device=self.dev)
        lat = torch.empty(B, n, self.H, self.rank, dtype=torch.float16, device=self.dev)
        out = torch.empty(B, n, self.H, self.v, dtype=torch.float16, device=self.dev)
        mkv.mkv_latent_absorb(self.cfg, q.data_ptr(), self.w_kv.data_ptr(), n, qa.data_ptr())
        mkv.mkv_latent_attention(self.cfg, qa.data_ptr(), self.cache.c, rows.data_ptr(), mask.data_ptr(), n,
                                 lat.data_ptr(), self.ws.data_ptr(), self.ws_bytes)
        mkv.mkv_latent_project(self.cfg, lat.data_ptr(), self.w_kv.data_ptr(), n, out.data_ptr())
        return self._logits(x, out), rows

    def commit(self, rows, path, accepted):
        mkv.mkv_latent_commit(self.cfg, rows.data_ptr(), path.data_ptr(), accepted.data_ptr(), rows.shape[1],
                              self.cache.c)


def speculative(model, prompt, steps):
    """Decodes `steps` passes with the draft tree; the accepted tokens of each entry."""
    B, n, dev = model.B, len(PARENT), model.dev
    mask = torch.tensor([tree_mask(PARENT)] * B, dtype=torch.int64, device=dev)
    depth = torch.tensor(DEPTH, device=dev)
    last = model.prefill(prompt).argmax(-1)
    said = [[int(t)] for t in last.tolist()]
    for _ in range(steps):
        tree = torch.empty(B, n, dtype=torch.int64, device=dev)
        tree[:, 0] = last
        for j in range(1, n):
            tree[:, j] = model.guess(tree[:, PARENT[j]], 2)[:, RANK[j]]
        pos = model.cache.t["T_len"].long()[:, None] + depth
        logits, rows = model.attend(tree, pos, mask)
        best = logits.argmax(-1).cpu().numpy()
        drafted = tree.cpu().numpy()
        path = np.zeros((B, n), dtype=np.int32)
        accepted = np.ones(B, dtype=np.int32)
        for b in range(B):
            at = 0
            while True:                    # follow the branch that the model agrees with
                nxt = [j for j in range(1, n) if PARENT[j] == at and drafted[b, j] == best[b, at]]
                if not nxt:
                    break
                at = nxt[0]
                path[b, accepted[b]] = at
                accepted[b] += 1
                said[b].append(int(drafted[b, at]))
            said[b].append(int(best[b, at]))
        model.commit(rows, torch.from_numpy(path).to(dev), torch.from_numpy(accepted).to(dev))
        last = torch.tensor([s[-1] for s in said], device=dev)
    return said


def one_by_one(model, prompt, tokens):
    """Decodes `tokens` tokens an entry, one a pass."""
    mask = torch.ones(model.B, 1, dtype=torch.int64, device=model.dev)
    path = torch.zeros(model.B, 1, dtype=torch.int32, device=model.dev)
    one = torch.ones(model.B, dtype=torch.int32, device=model.dev)
    last = model.prefill(prompt).argmax(-1)
    said = [[int(t)] for t in last.tolist()]
    for _ in range(tokens - 1):
        logits, rows = model.attend(last[:, None], model.cache.t["T_len"].long()[:, None], mask)
        model.commit(rows, path, one)
        last = logits[:, 0].argmax(-1)
        for s, t in zip(said, last.tolist()):
            s.append(int(t))
    return said


def main(B=2, T=200, steps=12, seed=0):
    """Returns (tokens said with the draft, the same one by one, passes)."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    prompt = torch.randint(0, 512, (B, T), generator=g, device="cuda")
    capacity = T + 4 * steps + 8
    fast = speculative(Model(B, capacity, seed), prompt, steps)
    slow = one_by_one(Model(B, capacity, seed), prompt, max(len(s) for s in fast))
    assert mkv.mkv_get_status() == 0
    return fast, slow, steps


if __name__ == "__main__":
    fast, slow, steps = main()
    for b, (f, s) in enumerate(zip(fast, slow)):
        same = next((i for i, (x, y) in enumerate(zip(f, s)) if x != y), len(f))
        print(f"entry {b}: {len(f) - 1} tokens in {steps} passes ({(len(f) - 1) / steps:.2f} a pass), "
              f"the first {same} as one by one: {f[:12]} ...")

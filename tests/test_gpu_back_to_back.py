"""Calls enqueued one after another on one stream with one workspace, and on two streams at once: nothing is
synchronised in between, so an answer that is read or overwritten too early shows."""
import numpy as np
import pytest

import tree_latent_calls as calls
from gpu_util import torch_cuda
from latent_util import randn, to_mask, tree_masks

pytestmark = pytest.mark.gpu

ROUNDS = 6


class Tree:
    """16 drafted rows a key head over two long entries: their keys are shared by many CTAs and joined in a second kernel."""
    def __init__(self, rng):
        B, Hkv, G, D, self.n, T_cap = 2, 2, 4, 128, 4, 8200
        self.k, self.v = (randn(rng, (B, Hkv, T_cap, D), "fp16") for _ in range(2))
        self.q = [randn(rng, (B, self.n, Hkv * G, D), "fp16") for _ in range(ROUNDS)]
        self.new = [randn(rng, (B, self.n, Hkv, D), "fp16") for _ in range(ROUNDS)]
        self.mask = to_mask(tree_masks(rng, B, self.n))
        self.in_q, self.in_new = (x[0].clone() for x in (self.q, self.new))
        self.plan = calls.tree_plan(self.in_q, self.k, self.v, [8190, 5001])

    def out(self):
        import torch
        return torch.full_like(self.in_q, 3.0)

    def call(self, out, stream):
        calls.tree_call(self.plan, self.in_q, self.in_new, self.in_new, self.mask, out, stream)


class Latent:
    def __init__(self, rng):
        B, H, rank, self.n, T_cap = 2, 16, 512, 3, 8200
        self.rows = randn(rng, (B, T_cap, rank + 64), "bf16")
        self.q = [randn(rng, (B, self.n, H, rank + 64), "bf16") for _ in range(ROUNDS)]
        self.new = [randn(rng, (B, self.n, rank + 64), "bf16") for _ in range(ROUNDS)]
        self.mask = to_mask(tree_masks(rng, B, self.n))
        self.in_q, self.in_new = (x[0].clone() for x in (self.q, self.new))
        self.plan = calls.latent_plan("bf16", self.in_q, self.rows, [8190, 5001])

    def out(self):
        import torch
        return torch.full(self.in_q.shape[:3] + (self.in_q.shape[3] - 64,), 3.0, dtype=self.in_q.dtype, device="cuda")

    def call(self, out, stream):
        calls.latent_call(self.plan, self.in_q, self.in_new, self.mask, out, stream)


def _alone(op):
    """Every round's answer with a device synchronisation around it."""
    import torch
    outs = []
    for i in range(ROUNDS):
        op.in_q.copy_(op.q[i])
        op.in_new.copy_(op.new[i])
        outs.append(op.out())
        torch.cuda.synchronize()
        op.call(outs[-1], None)
        torch.cuda.synchronize()
    return outs


def _enqueue(op, stream, outs):
    """All rounds: a kernel writes the inputs, the call reads them, and the next round's kernel overwrites them."""
    import torch
    with torch.cuda.stream(stream):
        for i in range(ROUNDS):
            torch.mul(op.q[i], 1.0, out=op.in_q)
            torch.mul(op.new[i], 1.0, out=op.in_new)
            op.call(outs[i], None if i % 2 else stream.cuda_stream)
            if i == ROUNDS // 2:
                op.call(outs[i], None)            # two calls with nothing in between


@pytest.mark.parametrize("kind", [Tree, Latent])
def test_one_stream_one_workspace(kind):
    torch = torch_cuda()
    op = kind(np.random.default_rng(7))
    want, outs, stream = _alone(op), [op.out() for _ in range(ROUNDS)], torch.cuda.Stream()
    torch.cuda.synchronize()
    _enqueue(op, stream, outs)
    stream.synchronize()
    for i, (a, b) in enumerate(zip(outs, want)):
        assert torch.equal(a, b), f"call {i}"


@pytest.mark.parametrize("kinds", [(Tree, Tree), (Latent, Latent), (Tree, Latent)])
def test_two_streams_at_once(kinds):
    torch = torch_cuda()
    ops = [kind(np.random.default_rng(8 + i)) for i, kind in enumerate(kinds)]
    want, outs = [_alone(op) for op in ops], [[op.out() for _ in range(ROUNDS)] for op in ops]
    streams = [torch.cuda.Stream() for _ in ops]
    torch.cuda.synchronize()
    for op, stream, out in zip(ops, streams, outs):
        _enqueue(op, stream, out)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(a, b) for a, b in zip(o, w))

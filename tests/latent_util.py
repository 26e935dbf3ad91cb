"""Helpers of the tree and latent GPU tests: inputs, and elementwise tolerances from the number formats.

With u the unit roundoff of the 16-bit type (2^-11 for fp16, 2^-8 for bf16), a kernel that rounds the
softmax weights and the output once each is off by at most
    u * mean|v| (weights)  +  u * |out| (output)  +  2 d * mean|v| (scores),
where mean|v| is the weighted mean of |v| and d bounds the error of a score in nats: 2^-22 of the sum of
|q k| scale per 16 products accumulated in fp32 (tensor cores may truncate), about 1e-4 for the inputs here.
What falls below the 16-bit type's normal range is off by at most half its smallest subnormal.
"""
import numpy as np

U = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp16": 2.0 ** -24, "bf16": 2.0 ** -126}
SCORE = 1.5e-4


def torch_dtype(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float16


def randn(rng, shape, dtype, dev="cuda", std=1.0):
    """Standard normals rounded to the type, on the device."""
    import torch
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch_dtype(dtype)).to(dev)


def f64(t):
    return t.detach().double().cpu().numpy()


def check_attention(got, ref, mag, dtype, what=""):
    got = f64(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    tol = (U[dtype] + 2 * SCORE) * mag + U[dtype] * np.abs(ref) + TINY[dtype]
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.abs(got - ref).max():.3e}, " \
                          f"first at {np.argwhere(bad)[0].tolist()}"


def check_product(got, ref, mag, dtype, what=""):
    """A product rounded once: u |out| plus 2^-18 of the sum of |x w| for the fp32 accumulation."""
    got = f64(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    tol = U[dtype] * np.abs(ref) + 2.0 ** -18 * mag + TINY[dtype]
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.abs(got - ref).max():.3e}"


def tree_masks(rng, B, n):
    """Random trees: token j sees itself and its ancestors."""
    m = np.zeros((B, n), dtype=np.uint64)
    for b in range(B):
        for j in range(n):
            p = int(rng.integers(-1, j)) if j else -1
            m[b, j] = np.uint64(1 << j) | (m[b, p] if p >= 0 else np.uint64(0))
    return m


def to_mask(m, dev="cuda"):
    import torch
    return torch.from_numpy(m.view(np.int64)).to(dev)

"""GPU parity of rotary positions: tables, both layouts, part of a head, strides, in place, and the gradient."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import paged as P
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import TINY, U, f64, randn, torch_dtype
from paged_util import KINDS, LAYOUTS, device, seeded

pytestmark = pytest.mark.gpu

SCALINGS = {
    "plain": {},
    "linear": dict(factor=4.0),
    "bands": dict(theta=500000.0, factor=8.0, low=1.0, high=4.0, context=8192),
    "ramp": dict(factor=16.0, low=1.0, high=32.0, context=4096),
}
CODES = {"plain": mkv.MKV_ROPE_PLAIN, "linear": mkv.MKV_ROPE_LINEAR, "bands": mkv.MKV_ROPE_BANDS, "ramp": mkv.MKV_ROPE_RAMP}


def _magnitude(scaling):
    return 0.1 * np.log(16.0) + 1.0 if scaling == "ramp" else 1.0


def _cfg(D, rot, layout, scaling, **kw):
    return mkv.rope_config(D, rot_dim=rot, layout=LAYOUTS[layout], scaling=CODES[scaling], **{**SCALINGS[scaling], **kw})


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("rot", [2, 32, 128, 250])
def test_table(scaling, rot):
    torch_cuda()
    n = 5003
    t = f64(caches.rope_table(_cfg(256, rot, "half", scaling), n))
    ref = P.table(np.arange(n), P.frequencies(rot, scaling=scaling, **SCALINGS[scaling]), _magnitude(scaling))
    # one rounding to fp32; angles up to 5003 in fp64 are off by a few 2^-53 of their size (2^-39)
    assert np.abs(t - ref).max() <= 2.0 ** -24 * _magnitude(scaling) + 2.0 ** -38


def test_table_far_positions_and_own_magnitude():
    torch_cuda()
    n = 1 << 20
    t = f64(caches.rope_table(_cfg(64, 64, "half", "plain", magnitude=2.5), n)[-64:])
    ref = P.table(np.arange(n - 64, n), P.frequencies(64), 2.5)
    assert np.abs(t - ref).max() <= 2.5 * (2.0 ** -24 + 2.0 ** -31)


def _run(cfg, dtype, x, pos, heads, table, out=None, transposed=False, x_stride=0, out_stride=0, stream=None):
    torch = torch_cuda()
    n = len(pos)
    out = torch.empty(n, heads, cfg.D, dtype=x.dtype, device=x.device) if out is None else out
    mkv.mkv_rope_apply(cfg, KINDS[dtype], x.data_ptr(), x_stride, pos.data_ptr(), n, heads, table.data_ptr(), table.shape[0],
                       transposed, out.data_ptr(), out_stride, stream)
    return out


def _check(x, pos, table, layout, got, dtype, transposed=False, what=""):
    cs = f64(table)[pos.cpu().numpy()]
    if transposed:
        cs = cs * np.array([1.0, -1.0])
    ref = P.rotate(f64(x), cs, layout)
    # fp32: two products and their sum are rounded, each by 2^-24 of |x c| + |y s| at most, which is no more than
    # (|x| + |y|) max(|c|, |s|): three of them are below 2^-22 of that
    r = 2 * cs.shape[1]
    i0 = np.arange(r // 2) if layout == "half" else np.arange(0, r, 2)
    i1 = i0 + r // 2 if layout == "half" else i0 + 1
    size = np.zeros_like(ref)
    size[..., i0] = size[..., i1] = (np.abs(f64(x))[..., i0] + np.abs(f64(x))[..., i1]) * np.abs(cs).max(-1)[:, None, :]
    err = np.abs(f64(got) - ref)
    tol = U[dtype] * (np.abs(ref) + 2.0 ** -22 * size) + 2.0 ** -22 * size + TINY[dtype]
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} off, worst {err.max():.3e}, first at {np.argwhere(bad)[0].tolist()}"


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("D,rot", [(128, 128), (64, 32), (80, 48), (256, 256), (256, 16), (6, 4), (40, 40), (2, 2)])
@pytest.mark.parametrize("n,heads", [(1, 1), (3, 40), (257, 7)])
def test_apply(dtype, layout, D, rot, n, heads):
    torch = torch_cuda()
    rng = seeded("apply", dtype, layout, D, rot, n, heads)
    cfg = _cfg(D, rot, layout, "plain")
    table = caches.rope_table(cfg, 4096)
    x = randn(rng, (n, heads, D), dtype)
    pos = device(rng.integers(0, 4096, n).astype(np.int32))
    for transposed in (False, True):
        _check(x, pos, table, layout, _run(cfg, dtype, x, pos, heads, table, transposed=transposed), dtype, transposed)
    inplace = x.clone()
    _run(cfg, dtype, inplace, pos, heads, table, out=inplace)
    assert torch.equal(inplace, _run(cfg, dtype, x, pos, heads, table))
    assert mkv.mkv_get_status() == 0


@pytest.mark.parametrize("n,heads", [(5, 3), (20000, 16)])
@pytest.mark.parametrize("extra,shift", [(0, 0), (16, 8), (13, 0), (8, 1)])
def test_strides_and_alignment(n, heads, extra, shift):
    """Heads within wider rows, rows that begin anywhere: the same numbers, and nothing written beside them."""
    torch = torch_cuda()
    D, rot = 64, 32
    rng = seeded("strides", n, heads, extra, shift)
    cfg = _cfg(D, rot, "half", "plain")
    table = caches.rope_table(cfg, 1000)
    row = heads * D + extra
    xs = randn(rng, (n * row + 32,), "bf16")
    pos = device(rng.integers(0, 1000, n).astype(np.int32))
    x = xs[shift:shift + n * row].view(n, row)[:, :heads * D].reshape(n, heads, D)
    buf = torch.full((n * row + 32,), 7.0, dtype=torch.bfloat16, device="cuda")
    flat = buf[shift:]
    mkv.mkv_rope_apply(cfg, mkv.MKV_BF16, xs.data_ptr() + 2 * shift, row, pos.data_ptr(), n, heads, table.data_ptr(), 1000, 0,
                       flat.data_ptr(), row)
    got = flat[:n * row].view(n, row)
    assert torch.equal(got[:, :heads * D].reshape(n, heads, D), _run(cfg, "bf16", x.contiguous(), pos, heads, table))
    assert (got[:, heads * D:] == 7).all() and (buf[:shift] == 7).all() and (flat[n * row:] == 7).all()


def test_table_at_eight_bytes():
    """A table that is not 16-byte aligned takes the narrow path, with the same results."""
    torch = torch_cuda()
    cfg = _cfg(64, 64, "half", "plain")
    t = caches.rope_table(cfg, 512)
    odd = torch.empty(t.numel() + 2, device="cuda")
    odd[2:].copy_(t.flatten())
    rng = seeded("eight")
    x, pos = randn(rng, (33, 4, 64), "fp16"), device(rng.integers(0, 512, 33).astype(np.int32))
    out = torch.empty_like(x)
    mkv.mkv_rope_apply(cfg, mkv.MKV_F16, x.data_ptr(), 0, pos.data_ptr(), 33, 4, odd.data_ptr() + 8, 512, 0, out.data_ptr(), 0)
    assert torch.equal(out, _run(cfg, "fp16", x, pos, 4, t))


def test_positions_outside_the_table():
    torch = torch_cuda()
    cfg = _cfg(64, 64, "half", "plain")
    table = caches.rope_table(cfg, 100)
    x = randn(seeded("outside"), (4, 2, 64), "fp16")
    got = _run(cfg, "fp16", x, torch.tensor([-1, 0, 99, 100], dtype=torch.int32, device="cuda"), 2, table)
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_BAD_INDEX
    near = _run(cfg, "fp16", x, torch.tensor([0, 0, 99, 99], dtype=torch.int32, device="cuda"), 2, table)
    assert torch.equal(got, near) and mkv.mkv_get_status() == 0


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_transposed_is_the_gradient(layout):
    """<rope(x + h d) - rope(x - h d), g> / 2 h = <d, rope^T(g)>, in the formula and by differences."""
    torch_cuda()
    cfg = _cfg(64, 32, layout, "ramp")
    table = caches.rope_table(cfg, 300)
    rng = seeded("gradient", layout)
    x, g, d = (randn(rng, (9, 3, 64), "fp16") for _ in range(3))
    pos = device(rng.integers(0, 300, 9).astype(np.int32))
    cs = f64(table)[pos.cpu().numpy()]
    gx = f64(_run(cfg, "fp16", g, pos, 3, table, transposed=True))
    want = P.rotate(f64(g), cs * np.array([1.0, -1.0]), layout)
    assert np.abs(gx - want).max() <= U["fp16"] * np.abs(want).max() + 2.0 ** -20
    # differences: powers of two keep x +- d / 2 within one rounding of fp16 each
    up, down = (_run(cfg, "fp16", (x + s * d), pos, 3, table) for s in (0.5, -0.5))
    slope = ((f64(up) - f64(down)) * f64(g)).sum()
    step = f64(x + 0.5 * d) - f64(x - 0.5 * d)
    # outputs up to about 8 are off by 2^-11 of themselves each, in 1728 products with |g|
    tol = U["fp16"] * ((np.abs(f64(up)) + np.abs(f64(down))) * np.abs(f64(g))).sum() + U["fp16"] * (np.abs(step) * np.abs(gx)).sum()
    assert abs(slope - (step * want).sum()) <= tol + 1e-6


def test_streams_and_graphs():
    torch = torch_cuda()
    cfg = _cfg(128, 128, "half", "plain")
    table = caches.rope_table(cfg, 4096)
    rng = seeded("graph")
    x, pos = randn(rng, (64, 8, 128), "bf16"), device(rng.integers(0, 4096, 64).astype(np.int32))
    want = _run(cfg, "bf16", x, pos, 8, table)
    out = torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _run(cfg, "bf16", x, pos, 8, table, out=out, stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)

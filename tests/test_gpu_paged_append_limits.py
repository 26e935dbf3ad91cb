"""GPU parity of the paged append where values are not finite, rotations overflow, or scales reach their ends: codes, scales,
lengths and flags, bit for bit."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv

from gpu_util import torch_cuda
from paged_util import device
from test_gpu_paged_append import Case

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
every = pytest.mark.parametrize("fmt", ["e4m3", "int8"])
rotated = pytest.mark.parametrize("layout,rot", [("half", 0), ("half", 128), ("pairs", 128), ("pairs", 48)])
# units of a warp and of a CTA, of empty pages, of one that holds tokens, and of several
pages = pytest.mark.parametrize("page,held,new", [(16, 0, 3), (16, 13, 2), (16, 9, 40), (64, 0, 40), (64, 20, 40), (128, 100, 150)])


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@every
@rotated
@pages
def test_not_finite(dtype, fmt, layout, rot, page, held, new):
    """Infinities as the largest code, NaN as zero, scales by the finite values; what a rotation makes of them too."""
    for name, where, value in (("v", (1, 0, 3), INF), ("v", (0, 1, 127), NAN), ("k", (1, 0, 5), INF), ("k", (0, 1, 100), -INF),
                               ("k", (new - 1, 1, 17), NAN), ("k", (1, 1, 0), -INF)):
        c = Case(dtype, fmt, 1, 2, 2, 128, page, [held], [new], rot=rot, layout=layout, key=(name, where))
        getattr(c, name)[where] = value
        c.run()
        c.check(flags=mkv.MKV_FLAG_NOT_FINITE, what=f"{name} {where} {value}")


@every
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pages
def test_rotation_overflows(fmt, layout, page, held, new):
    """Finite keys near the type's largest number whose rotation is not: sums and differences of products beyond fp32."""
    c = Case("bf16", fmt, 1, 2, 2, 128, page, [held], [new], layout=layout)
    c.k[:, 0] = 3.3e38
    c.k[1, 1] = -3.3e38
    c.run()
    c.check(flags=mkv.MKV_FLAG_NOT_FINITE)


@every
@pages
def test_zeros_of_either_sign(fmt, page, held, new):
    c = Case("bf16", fmt, 1, 2, 2, 128, page, [held], [new])
    c.k[:] = 0.0
    c.v[:, 0] = -0.0
    c.run()
    c.check()


def _held_page(was, dtype="bf16", fmt="int8", page=16, value=3.3e38):
    c = Case(dtype, fmt, 1, 2, 2, 64, page, [page // 2], [3], rot=0)
    for name, x in (("k_scale", c.hc.ks), ("v_scale", c.hc.vs)):
        x[:] = was
        c.hc.cache.t[name].copy_(device(x))
    c.k[:, 0] = value
    c.v[:, 1] = -value
    return c


@every
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("was", [1.5 * 2.0 ** 120, 2.0 ** 120, 1.25 * 2.0 ** 119, 1.5 * 2.0 ** 125, 1.5 * 2.0 ** -126, 2.0 ** -101])
def test_scales_at_their_ends(fmt, page, was):
    """A page's scale is only ever raised: one above the largest that an append gives stays, with the codes that it has."""
    torch = torch_cuda()
    c = _held_page(np.float32(was), fmt=fmt, page=page)
    held = {x: c.hc.cache.t[x].clone() for x in ("k", "v")}
    c.run()
    c.check()
    pid = int(c.hc.table[0, 0])
    for x, name in (("k", "k_scale"), ("v", "v_scale")):
        assert (c.hc.cache.t[name][pid] >= np.float32(was)).all()
        if was > 2.0 ** 120:
            assert torch.equal(c.hc.cache.t[x][pid, :, :page // 2].view(torch.uint8), held[x][pid, :, :page // 2].view(torch.uint8))

"""GPU parity of attention over 8-bit pages where more than 32 query rows share a key head: prompts, their chunks, many
drafted tokens."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv

from gpu_util import torch_cuda
from paged_util import check_attention, device
from test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_shapes(dtype, fmt, D, page):
    """Whole prompts and chunks behind a beginning, ends within pages and tiles, entries of one row and of none."""
    lens = [1, 33, 100, 128, 129, 300, 511, 40]
    new = [1, 33, 64, 128, 100, 300, 37, 0]
    c = Case(dtype, fmt, 4, 2, D, page, lens, new)
    c.run()
    c.check()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (7, 1), (8, 8), (32, 1), (24, 3)])
def test_heads(Hq, Hkv):
    c = Case("fp16", "e4m3", Hq, Hkv, 128, 32, [200, 65], [150, 34])
    c.run()
    c.check()


@pytest.mark.parametrize("n", [33, 64, 129])
def test_without_start(n):
    c = Case("bf16", "int8", 8, 2, 64, 16, [n, n + 100, 400], [n, n, n], ragged=False)
    c.run()
    c.check()


@pytest.mark.parametrize("T,n", [(4001, 40), (9000, 64), (2500, 300)])
def test_long_histories_shared_out(T, n):
    """Few units: the tokens of each are shared out, some parts without any."""
    c = Case("fp16", "int8", 4, 2, 128, 64, [T, 70], [n, 60])
    c.run()
    c.check()


def test_many_units():
    """More units than SMs: nothing is shared out."""
    c = Case("bf16", "e4m3", 16, 8, 64, 16, [150 + 7 * b for b in range(24)], [100 + b for b in range(24)])
    c.run()
    c.check()


def test_rows_before_the_first_position_and_empty_entries():
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, 16, [0, 3, 50], [20, 60, 40])
    c.run()
    c.check()
    assert (c.out[:20] == 0).all() and (c.out[20:77] == 0).all() and torch.isfinite(c.out).all()


def test_scales_far_apart():
    c = Case("bf16", "e4m3", 8, 2, 64, 16, [500, 90], [100, 40], wild=30)
    c.run()
    c.check()


def test_page_of_zeros_has_the_least_scale():
    c = Case("bf16", "int8", 4, 2, 64, 16, [300, 40], [100, 17])
    for b in range(2):
        pid = c.hc.table[b, 1]
        c.hc.v[pid], c.hc.vs[pid] = 0, 2.0 ** -100
    c.hc.cache.t["v"].copy_(device(c.hc.v))
    c.hc.cache.t["v_scale"].copy_(device(c.hc.vs))
    c.run()
    c.check()


def test_large_and_small_queries():
    big = Case("bf16", "e4m3", 4, 2, 64, 16, [100, 53], [50, 52], std=2.0 ** 40, scale=2.0 ** -43)
    big.run()
    big.check()
    small = Case("bf16", "int8", 4, 2, 128, 16, [100, 53], [50, 52], std=2.0 ** -60, scale=2.0 ** 56)
    small.run()
    small.check()


def test_infinite_queries_stay_in_their_rows():
    """NaN in the row itself; the others are right (when a maximum is raised is a warp's common choice, so they may be
    rounded another way)."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 4, 2, 64, 16, [100, 60], [50, 60])
    want, was = c.run().clone(), c.q[7, 1, 5].clone()
    c.q[7, 1, 5] = float("inf")
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[7, 1]).all()
    c.q[7, 1, 5] = was
    c.out[7, 1] = want[7, 1]
    c.check()


def test_what_lies_behind_the_length_is_not_seen():
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, 64, [170, 70], [50, 9])
    want = c.run().clone()
    for b, t in enumerate(c.hc.lens):
        pid = int(c.hc.table[b, t // 64])
        c.hc.cache.t["k"].view(torch.uint8)[pid, :, t % 64:] = 0x7f
        c.hc.cache.t["v"].view(torch.uint8)[pid, :, t % 64:] = 0xff
    c.run()
    c.check()
    assert bool((c.out == want).all())


def test_pages_outside_the_pool_are_not_seen():
    for bad in (-1, 1 << 30):
        c = Case("fp16", "e4m3", 8, 2, 64, 16, [300, 50], [40, 33])
        c.hc.cache.t["page_table"][0, 3] = bad
        c.run()
        hole = lambda b, t: (np.arange(t) // 16 != 3) if b == 0 else np.ones(t, bool)
        c.check(flags=mkv.MKV_FLAG_BAD_INDEX, seen=hole)


def test_too_many_rows_of_an_entry():
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 4, 2, 64, 16, [140, 140, 140], [40, 70, 1])
    c.most = 40
    c.run()
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_BAD_INDEX
    assert (c.out[40:110] == 3).all()
    check_attention(c.hc, c.q, c.starts, c.out, c.dtype, entries=(0, 2))


def test_strides():
    torch = torch_cuda()
    c = Case("bf16", "int8", 6, 2, 128, 32, [100, 3, 64], [52, 1, 35])
    want = c.run()[:c.n].clone()
    wide = torch.full((c.n, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :6] = c.q[:c.n]
    out = torch.full((c.n, 7, 128), 4.0, dtype=torch.bfloat16, device="cuda")
    mkv.mkv_paged_attention(c.cfg, wide.data_ptr(), 8 * 128, c.start.data_ptr(), c.n, c.most, c.hc.cache.c, out.data_ptr(),
                            7 * 128, c.ws.data_ptr(), c.nws)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :6], want) and (out[:, 6] == 4).all()


def test_same_rows_by_both_kernels():
    """The same newest tokens, as few rows and as the end of a chunk, within both kernels' error."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, 16, [900], [64])
    c.run()
    c.check()
    last = Case("fp16", "e4m3", 8, 2, 128, 16, [900], [4], key=1)
    last.hc, last.q = c.hc, c.q[60:].contiguous()
    last.run()
    last.check()
    assert torch.allclose(last.out[:4].float(), c.out[60:64].float(), atol=2e-3)


def test_graphs_and_streams():
    torch = torch_cuda()
    cases = [Case("fp16", "e4m3", 8, 2, 128, 16, [3000, 777], [40, 100]), Case("fp16", "e4m3", 8, 2, 128, 16, [500, 400], [400, 2])]
    ws, nws = max(((c.ws, c.nws) for c in cases), key=lambda x: x[1])
    own = [(c.ws, c.nws) for c in cases]
    want, graphs = [], []
    for c in cases:
        c.ws, c.nws = ws, nws
        want.append(c.run().clone())
    for c in cases:
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            c.run(torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for _ in range(4):
        for c, g, w in zip(cases, graphs, want):
            c.out[:c.n].fill_(0)
            g.replay()
            assert torch.equal(c.out, w)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for c, (w, n) in zip(cases, own):
        c.ws, c.nws = (w.clone(), n)
    torch.cuda.synchronize()
    for _ in range(6):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.out[:c.n].fill_(0)
                c.run(s.cuda_stream)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c.out, w)
    assert mkv.mkv_get_status() == 0

"""GPU parity of attention over 8-bit pages."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import f64, randn, torch_dtype
from paged_util import FORMATS, KINDS, HostCache, check_attention, device, seeded

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, dtype="fp16", fmt="e4m3", Hq=8, Hkv=2, D=128, page=16, lens=(5, 40), new=(1, 1), ragged=True,
                 key=0, max_pages=None, std=1.0, tail=2, scale=0.0, **cache):
        torch = torch_cuda()
        rng = seeded("attend", dtype, fmt, Hq, Hkv, D, page, tuple(lens), tuple(new), key)
        B = len(lens)
        self.dtype, self.ragged, self.new, self.scale = dtype, ragged, list(new), scale or None
        self.cfg = mkv.paged_config(KINDS[dtype], FORMATS[fmt], B, Hq, Hkv, D, page, softmax_scale=scale)
        self.hc = HostCache(rng, self.cfg, fmt, lens, max_pages or max(1, -(-max(lens) // page)) + 1, **cache)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.n, self.most = int(self.starts[-1]), max(new)
        self.q = randn(rng, (self.n + tail, Hq, D), dtype, std=std)
        self.start = device(self.starts) if ragged else None
        self.out = torch.full((self.n + tail, Hq, D), 3.0, dtype=torch_dtype(dtype), device="cuda")
        self.ws, self.nws = caches.paged_workspace(self.cfg, self.n, self.most)
        self.ws[16384:].fill_(255)

    def run(self, stream=None, out=None):
        torch_cuda()
        mkv.mkv_paged_attention(self.cfg, self.q.data_ptr(), 0, self.start.data_ptr() if self.ragged else 0, self.n, self.most,
                                self.hc.cache.c, (self.out if out is None else out).data_ptr(), 0, self.ws.data_ptr(),
                                self.nws, stream)
        return self.out

    def check(self, flags=0, what="", **kw):
        torch = torch_cuda()
        torch.cuda.synchronize()
        assert mkv.mkv_get_status() == flags, what
        assert (self.ws[:16384] == 0).all(), what
        assert (self.out[self.n:] == 3).all(), what
        check_attention(self.hc, self.q, self.starts, self.out, self.dtype, self.scale, what, **kw)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (14, 2), (32, 1)])
def test_single_tokens(dtype, fmt, D, page, Hq, Hkv):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 333]
    c = Case(dtype, fmt, Hq, Hkv, D, page, lens, [1] * len(lens), ragged=page != 32)
    c.run()
    c.check()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,new", [(4, 4, [2, 8, 5, 16, 1]), (8, 2, [8, 3, 1, 0, 8]), (3, 1, [10, 1, 9, 4, 7]),
                                        (16, 2, [4, 2, 3, 4, 1]), (6, 6, [32, 17, 31, 30, 9])])
def test_drafted_tokens(dtype, D, Hq, Hkv, new):
    """Causal among themselves, more rows than one block of eight, entries without any."""
    for page, fmt in ((16, "e4m3"), (64, "int8")):
        c = Case(dtype, fmt, Hq, Hkv, D, page, [40, 64, 65, 130, 300], new)
        c.run()
        c.check()


@pytest.mark.parametrize("T,page", [(1000, 16), (8192, 64), (30011, 32)])
@pytest.mark.parametrize("n", [1, 8])
def test_long_contexts_split(T, page, n):
    """Units shared by several CTAs, and CTAs that hold several units."""
    c = Case("fp16", "int8", 8, 2, 128, page, [T, T // 2 + 1, 3, T // 3], [n, n, min(n, 3), n])
    c.run()
    c.check()


def test_many_entries():
    rng = seeded("entries")
    lens = rng.integers(1, 200, 100).tolist()
    c = Case("bf16", "e4m3", 8, 4, 64, 16, lens, [1] * 100)
    c.run()
    c.check()


def test_rows_before_the_first_position_and_empty_entries():
    """More new tokens than the entry holds: the rows before position 0 get zeros; so do all rows of an empty entry."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, 16, [0, 3, 20], [2, 5, 1], ragged=True)
    c.run()
    c.check()
    assert (c.out[:2] == 0).all() and (c.out[2:4] == 0).all() and not (c.out[4:7] == 0).all(-1).any()
    assert torch.isfinite(c.out).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [64, 128])
def test_every_code(fmt, D):
    """A value row that holds every code, met alone: outputs are the codes' values; and keys of every code."""
    torch = torch_cuda()
    c = Case("fp16", fmt, 2, 2, D, 16, [1] * (256 // D), [1] * (256 // D))
    codes = np.arange(256, dtype=np.uint8)
    if fmt == "e4m3":
        codes[[0x7f, 0xff]] = 0                           # (NaN)
    codes = codes.reshape(-1, D)
    for b in range(256 // D):
        for h in range(2):
            c.hc.v[c.hc.table[b, 0], h, 0] = codes[b].view(c.hc.v.dtype)
            c.hc.k[c.hc.table[b, 0], h, 0] = codes[b].view(c.hc.k.dtype)
    for name in ("k", "v"):
        t = c.hc.cache.t[name]
        t.copy_(device(getattr(c.hc, name)).view(t.dtype))
    c.hc.ks[:] = c.hc.vs[:] = 1.0
    for name in ("k_scale", "v_scale"):
        c.hc.cache.t[name].fill_(1.0)
    c.run()
    torch.cuda.synchronize()
    for b in range(256 // D):
        _, V = c.hc.tokens(b, 0, 1)
        assert np.array_equal(f64(c.out[b, 0]), V[0])


def test_scales_far_apart():
    """Pages whose value scales differ by 2^60: each row keeps full precision at the size of what it attends to."""
    c = Case("bf16", "e4m3", 8, 2, 64, 16, [500, 90], [1, 4], wild=30)
    c.run()
    c.check()


def test_page_of_zeros_has_the_least_scale():
    c = Case("bf16", "int8", 4, 2, 64, 16, [64, 40], [1, 1])
    for b in range(2):
        pid = c.hc.table[b, 1]
        c.hc.v[pid], c.hc.vs[pid] = 0, 2.0 ** -100
    c.hc.cache.t["v"].copy_(device(c.hc.v))
    c.hc.cache.t["v_scale"].copy_(device(c.hc.vs))
    c.run()
    c.check()


def test_large_and_small_queries():
    """bf16 queries beyond fp16's range, both ways (a small scale keeps their scores of usual size)."""
    big = Case("bf16", "e4m3", 4, 2, 64, 16, [100, 3], [1, 2], std=2.0 ** 40, scale=2.0 ** -43)
    big.run()
    big.check()
    small = Case("bf16", "int8", 4, 2, 128, 16, [100, 3], [1, 2], std=2.0 ** -60, scale=2.0 ** 56)
    small.run()
    small.check()


def test_scores_that_leave_no_weight():
    """Infinite queries: NaN where the formula has it, and only there."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 4, 2, 64, 16, [100, 40], [1, 1])
    want = c.run().clone()
    c.q[0, 1, 5] = float("inf")
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[0, 1]).all()
    keep = torch.ones(c.n, 4, dtype=torch.bool, device="cuda")
    keep[0, 1] = False
    assert torch.equal(c.out[:c.n][keep], want[:c.n][keep])


def test_what_lies_behind_the_length_is_not_seen():
    c = Case("fp16", "e4m3", 8, 2, 128, 64, [70, 1], [2, 1])
    want = c.run().clone()
    for b, t in enumerate(c.hc.lens):
        pid = c.hc.table[b, t // 64]
        c.hc.cache.t["k"].view(__import__("torch").uint8)[int(pid), :, t % 64:] = 0x7f
        c.hc.cache.t["v"].view(__import__("torch").uint8)[int(pid), :, t % 64:] = 0xff
    c.run()
    c.check()
    assert bool((c.out == want).all())


def test_pages_outside_the_pool_are_not_seen():
    for bad in (-1, 1 << 30):
        c = Case("fp16", "e4m3", 8, 2, 64, 16, [100, 50], [1, 3])
        keep = c.hc.table[0, 3]
        c.hc.cache.t["page_table"][0, 3] = bad
        c.run()
        hole = lambda b, t: (np.arange(t) // 16 != 3) if b == 0 else np.ones(t, bool)
        c.check(flags=mkv.MKV_FLAG_BAD_INDEX, seen=hole)
        assert keep >= 0


def test_too_many_rows_of_an_entry():
    """An entry with more than max_rows rows is left out; the others are as they were."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 4, 2, 64, 16, [40, 40, 40], [2, 3, 1])
    c.most = 2
    c.run()
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_BAD_INDEX
    assert (c.out[2:5] == 3).all()
    check_attention(c.hc, c.q, c.starts, c.out, c.dtype, entries=(0, 2))


def test_lengths_beyond_the_table():
    """A length beyond what the table can hold is taken as the table's."""
    c = Case("fp16", "e4m3", 4, 2, 64, 16, [64, 20], [1, 1], max_pages=4)
    c.hc.cache.t["T_len"][0] = 1000
    c.run()
    c.check()


def test_strides():
    torch = torch_cuda()
    c = Case("bf16", "int8", 6, 2, 128, 32, [100, 3, 64], [2, 1, 5])
    want = c.run()[:c.n].clone()
    wide = torch.full((c.n, 8, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :6] = c.q[:c.n]
    out = torch.full((c.n, 7, 128), 4.0, dtype=torch.bfloat16, device="cuda")
    mkv.mkv_paged_attention(c.cfg, wide.data_ptr(), 8 * 128, c.start.data_ptr(), c.n, c.most, c.hc.cache.c, out.data_ptr(),
                            7 * 128, c.ws.data_ptr(), c.nws)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :6], want) and (out[:, 6] == 4).all()


def test_same_results_every_time_and_in_graphs():
    torch = torch_cuda()
    cases = [Case("fp16", "e4m3", 8, 2, 128, 16, [3000, 777], [1, 1]), Case("fp16", "e4m3", 8, 2, 128, 16, [500, 4000], [4, 2])]
    ws, nws = max(((c.ws, c.nws) for c in cases), key=lambda x: x[1])
    want = []
    for c in cases:
        c.ws, c.nws = ws, nws                             # (graphs that share a workspace, replayed in turn)
        want.append(c.run().clone())
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=side):
            c.run(torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for _ in range(5):
        for c, g, w in zip(cases, graphs, want):
            c.out[:c.n].fill_(0)
            g.replay()
            assert torch.equal(c.out, w)
    assert mkv.mkv_get_status() == 0


def test_two_streams_at_once():
    torch = torch_cuda()
    cases = [Case("fp16", "int8", 8, 2, 128, 16, [3000, 700], [1, 1], key=k) for k in range(2)]
    want = [c.run().clone() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.out[:c.n].fill_(0)
                c.run(s.cuda_stream)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c.out, w)

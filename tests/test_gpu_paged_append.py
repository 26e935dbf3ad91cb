"""GPU parity of the paged append: codes, scales and lengths bit for bit, rotated queries, refusals."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import paged as P
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import f64, randn, torch_dtype
from paged_util import FORMATS, KINDS, LAYOUTS, HostCache, device, seeded

pytestmark = pytest.mark.gpu


def _starts(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


class Case:
    def __init__(self, dtype="bf16", fmt="e4m3", B=2, Hq=8, Hkv=2, D=128, page=16, lens=(5, 40), new=(1, 1), rot=None,
                 layout="half", ragged=True, max_pages=None, pow2=True, pos=None, std=1.0, key=0, tail=0):
        torch = torch_cuda()
        self.rng = rng = seeded("append", dtype, fmt, B, Hq, Hkv, D, page, tuple(lens), tuple(new), rot, layout, key)
        self.dtype, self.fmt, self.new, self.layout, self.ragged = dtype, fmt, list(new), layout, ragged
        self.cfg = mkv.paged_config(KINDS[dtype], FORMATS[fmt], B, Hq, Hkv, D, page)
        most = max_pages or max(-(-(t + m) // page) for t, m in zip(lens, new)) + 1
        self.hc = HostCache(rng, self.cfg, fmt, lens, most, pow2=pow2)
        self.n = sum(new)
        width = Hq + 2 * Hkv
        self.qkv = randn(rng, (self.n + tail, width, D), dtype, std=std)
        self.q, self.k, self.v = self.qkv[:, :Hq], self.qkv[:, Hq:Hq + Hkv], self.qkv[:, Hq + Hkv:]
        self.row = width * D
        self.rot = D if rot is None else rot
        self.rope = mkv.rope_config(D, rot_dim=self.rot, layout=LAYOUTS[layout]) if self.rot else None
        self.T = max(max(t + m for t, m in zip(lens, new)), (max_pages or 0) * page) + 5
        self.table = caches.rope_table(self.rope, self.T) if self.rot else None
        self.start = device(_starts(new)) if ragged else None
        self.pos = device(np.asarray(pos, dtype=np.int32)) if pos is not None else None
        self.out = torch.full((self.n + tail, Hq, D), 3.0, dtype=torch_dtype(dtype), device="cuda")

    def run(self, stream=None):
        rows = mkv.paged_rows(self.n, start=self.start.data_ptr() if self.ragged else 0,
                              pos=self.pos.data_ptr() if self.pos is not None else 0, q=self.q.data_ptr(), q_stride=self.row,
                              k=self.k.data_ptr(), k_stride=self.row, v=self.v.data_ptr(), v_stride=self.row,
                              q_out=self.out.data_ptr())
        mkv.mkv_paged_append(self.cfg, self.rope, self.table.data_ptr() if self.rot else 0, self.T, rows, self.hc.cache.c,
                             stream)

    def expect(self, refused=()):
        """The oracle's pages, scales, lengths and queries."""
        hc, cfg, page = self.hc, self.cfg, self.hc.page
        st = _starts(self.new)
        f32 = lambda t: t.float().cpu().numpy()
        k, v, q = f32(self.k[:self.n]), f32(self.v[:self.n]), f32(self.q[:self.n])
        pos = np.concatenate([t + np.arange(m) for t, m in zip(hc.lens, self.new)]) if self.pos is None else \
            self.pos.cpu().numpy()
        if self.rot:
            cs = self.table.cpu().numpy()[np.clip(pos, 0, self.T - 1)]
            with np.errstate(invalid="ignore", over="ignore"):
                k, q = P.rotate(k, cs, self.layout), P.rotate(q, cs, self.layout)
        lens = hc.lens.copy()
        for b, m in enumerate(self.new):
            if b in refused or m == 0:
                continue
            t = int(hc.lens[b])
            for p in range(t // page, (t + m - 1) // page + 1):
                i0, i1 = max(0, p * page - t), min(m, (p + 1) * page - t)
                held, pid = max(0, t - p * page), hc.table[b, p]
                for h in range(cfg.Hkv):
                    for codes, scales, x in ((hc.k, hc.ks, k), (hc.v, hc.vs, v)):
                        scales[pid, h] = P.append_page(codes[pid, h], scales[pid, h], held, x[st[b] + i0:st[b] + i1, h],
                                                       self.fmt)
            lens[b] += m
        hc.lens = lens
        return q

    def check(self, refused=(), flags=0, what=""):
        torch = torch_cuda()
        q = self.expect(refused)
        torch.cuda.synchronize()
        assert mkv.mkv_get_status() == flags, what
        hc = self.hc
        assert hc.cache.t["T_len"].cpu().numpy().tolist() == hc.lens.tolist(), what
        assert (hc.cache.t["tickets"] == 0).all(), what
        for name, codes, scales in (("k", hc.k, hc.ks), ("v", hc.v, hc.vs)):
            assert np.array_equal(hc.cache.t[name + "_scale"].cpu().numpy(), scales), f"{what} {name} scales"
            got = hc.device_codes(name)
            assert np.array_equal(got, codes), f"{what} {name}: {int((got != codes).sum())} codes differ"
        want = torch.from_numpy(q).to(self.out.dtype).cuda()
        assert torch.equal(self.out[:self.n].nan_to_num(9.0), want.nan_to_num(9.0)), what
        assert (self.out[self.n:] == 3).all(), what


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_shapes(dtype, fmt, D, page):
    """Single tokens, some, and whole pages; pages that begin, go on and end; entries without any row."""
    lens = [0, 1, page - 1, page, 3 * page + 5, 77]
    for new in ([1] * 6, [0, 1, 2, 9, 3, 17], [page, page - 1, page + 1, 4 * page, 3, 200]):
        c = Case(dtype, fmt, 6, 6, 2, D, page, lens, new, tail=3)
        c.run()
        c.check(what=f"{new}")


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("layout,rot", [("half", 128), ("pairs", 128), ("half", 32), ("pairs", 48), ("half", 0)])
def test_rotations(fmt, layout, rot):
    c = Case("bf16", fmt, 3, 12, 3, 128, 32, [10, 0, 31], [2, 70, 33], rot=rot, layout=layout)
    c.run()
    c.check()


@pytest.mark.parametrize("n", [1, 5, 64, 130])
def test_without_start(n):
    """Every entry has n rows."""
    c = Case("fp16", "e4m3", 4, 8, 4, 64, 64, [0, 63, 64, 100], [n] * 4, ragged=False)
    c.run()
    c.check()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (40, 40), (96, 3), (7, 7), (21, 3)])
def test_heads(Hq, Hkv):
    for page, new in ((16, [1, 3]), (64, [100, 64])):
        c = Case("bf16", "int8", 2, Hq, Hkv, 64, page, [17, 0], new)
        c.run()
        c.check()


def test_many_entries():
    B = 300
    rng = seeded("many")
    lens, new = rng.integers(0, 60, B).tolist(), rng.integers(0, 7, B).tolist()
    c = Case("fp16", "int8", B, 4, 2, 64, 16, lens, new)
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("pow2", [True, False])
def test_page_keeps_or_raises_its_scale(fmt, pow2):
    """Small tokens leave a page's scale, large ones raise it and round its codes again; any positive scale may be there."""
    for std in (2.0 ** -6, 1.0, 40.0):
        c = Case("bf16", fmt, 2, 4, 4, 128, 32, [20, 7], [3, 1], pow2=pow2, std=std, key=std)
        c.run()
        c.check(what=f"std {std}")


def test_step_after_step():
    c = Case("bf16", "e4m3", 2, 4, 2, 64, 16, [0, 13], [1, 1], max_pages=4)
    for _ in range(20):
        c.run()
        c.check()
        c.qkv.mul_(1.25)


def test_own_positions():
    c = Case("bf16", "e4m3", 2, 4, 2, 64, 16, [3, 9], [4, 2], pos=[7, 1, 0, 14, 3, 2])
    c.run()
    c.check()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_zeros_tiny_and_huge(fmt):
    """Scales stay within 2^-100 .. 2^120; zeros have the least."""
    for value in (0.0, 2.0 ** -126, 2.0 ** -93, 3.0e38, -3.3e38):
        c = Case("bf16", fmt, 1, 2, 2, 64, 16, [0], [5], rot=0, key=value)
        c.qkv.fill_(value)
        c.run()
        c.check(what=str(value))


def test_not_finite():
    """Infinities are stored as the largest code, NaN as zero; the scale is that of the finite values."""
    for page, m in ((16, 3), (64, 40)):
        c = Case("bf16", "e4m3", 1, 2, 2, 64, page, [0], [m], rot=0)
        c.v[1, 0, 3] = float("inf")
        c.v[1, 1, 4] = float("-inf")
        c.k[2, 0, 5] = float("nan")
        c.run()
        c.check(flags=mkv.MKV_FLAG_NOT_FINITE)


def test_full_entries_are_refused_whole():
    c = Case("bf16", "e4m3", 3, 4, 2, 64, 16, [30, 30, 0], [2, 3, 32], max_pages=2)
    c.run()
    c.check(refused=(1,), flags=mkv.MKV_FLAG_CACHE_FULL)


def test_pages_outside_the_pool_are_refused_whole():
    for bad in (-1, 1 << 30):
        c = Case("bf16", "int8", 3, 4, 2, 64, 16, [10, 10, 10], [30, 30, 4])
        c.hc.table[1, 2] = bad
        c.hc.cache.t["page_table"].copy_(device(c.hc.table))
        c.run()
        c.check(refused=(1,), flags=mkv.MKV_FLAG_BAD_INDEX)


def test_queries_in_place_and_none():
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 2, 4, 2, 64, 16, [3, 9], [4, 2])
    before = c.qkv.clone()
    rows = mkv.paged_rows(c.n, start=c.start.data_ptr(), q=c.q.data_ptr(), q_stride=c.row, q_out=c.q.data_ptr(),
                          q_out_stride=c.row, k=c.k.data_ptr(), k_stride=c.row, v=c.v.data_ptr(), v_stride=c.row)
    mkv.mkv_paged_append(c.cfg, c.rope, c.table.data_ptr(), c.T, rows, c.hc.cache.c)
    torch.cuda.synchronize()
    c.out[:c.n].copy_(c.q)
    c.qkv.copy_(before)
    c.check()
    rows = mkv.paged_rows(c.n, start=c.start.data_ptr(), k=c.k.data_ptr(), k_stride=c.row, v=c.v.data_ptr(), v_stride=c.row)
    c.out.fill_(3.0)
    mkv.mkv_paged_append(c.cfg, c.rope, c.table.data_ptr(), c.T, rows, c.hc.cache.c)
    torch.cuda.synchronize()
    assert (c.out == 3).all()
    c.out[:c.n].copy_(torch.from_numpy(c.expect()).to(c.out.dtype))
    c.new = [0, 0]
    c.n = 0
    for name, codes in (("k", c.hc.k), ("v", c.hc.v)):
        assert np.array_equal(c.hc.device_codes(name), codes)


def test_captured_and_replayed():
    torch = torch_cuda()
    c = Case("bf16", "e4m3", 2, 4, 2, 64, 16, [0, 5], [1, 1], max_pages=4)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        c.run(torch.cuda.current_stream().cuda_stream)
    for _ in range(18):
        graph.replay()
        c.check()

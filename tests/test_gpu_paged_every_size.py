"""Attention over 8-bit pages at every number of rows that is computed in a way of its own: what can go wrong, at each."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv

from gpu_util import torch_cuda
from paged_util import check_attention, device
from test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu

# most new tokens of an entry, times 4 heads a group: 8, 32, 64, 120 and 280 query rows a key head
MOST = [2, 8, 16, 30, 70]
every = pytest.mark.parametrize("most", MOST)


def new_of(most, B):
    return [most if b == 0 else (most * (3 + 5 * b) // 7) % (most + 1) for b in range(B)]


@every
@pytest.mark.parametrize("page", [16, 128])
def test_missing_pages(most, page):
    """Pages outside the pool are not seen, the one with the newest tokens too; an entry without any gets NaN."""
    torch = torch_cuda()
    c = Case("bf16", "e4m3", 8, 2, 64, page, [700, 150, 260, 90], [most, 1, most, most])
    t = c.hc.cache.t["page_table"]
    t[0, 1], t[0, 5 if page == 128 else 40], t[2, 260 // page] = -1, 1 << 30, -7
    t[3] = -1
    c.run()
    gone = {0: (1, 5 if page == 128 else 40), 2: (260 // page,)}
    c.check(flags=mkv.MKV_FLAG_BAD_INDEX, entries=(0, 1, 2), seen=lambda b, n: ~np.isin(np.arange(n) // page, gone.get(b, ())))
    assert torch.isnan(c.out[c.starts[3]:c.n]).all()


@every
def test_too_many_rows(most):
    torch = torch_cuda()
    c = Case("fp16", "int8", 8, 2, 128, 16, [240, 240, 240], [most, most + 1, 1])
    c.most = most
    c.run()
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_BAD_INDEX
    assert (c.out[most:2 * most + 1] == 3).all()
    check_attention(c.hc, c.q, c.starts, c.out, c.dtype, entries=(0, 2))


@every
def test_rows_before_the_first_position(most):
    """Entries with fewer tokens than rows, with one and with none."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, 32, [0, 1, most - 1, 300], [most, most, most, most])
    c.run()
    c.check()
    assert (c.out[:2 * most - 1] == 0).all() and (c.out[2 * most] == 0).all()


@every
def test_scales_far_apart(most):
    c = Case("bf16", "e4m3", 8, 2, 64, 16, [500, 90, 300], new_of(most, 3), wild=30)
    c.run()
    c.check()


@every
@pytest.mark.parametrize("std,scale", [(2.0 ** 40, 2.0 ** -43), (2.0 ** -60, 2.0 ** 56)])
def test_large_and_small_queries(most, std, scale):
    c = Case("bf16", "int8", 8, 2, 64, 64, [400, 72], [most, most], std=std, scale=scale)
    c.run()
    c.check()


@every
def test_queries_not_finite(most):
    torch = torch_cuda()
    for x in (float("inf"), float("nan")):
        c = Case("bf16", "e4m3", 8, 2, 128, 16, [400, 72], [most, most])
        want, was = c.run().clone(), c.q[1, 3, 5].clone()
        c.q[1, 3, 5] = x
        c.run()
        torch.cuda.synchronize()
        assert torch.isnan(c.out[1, 3]).all()
        c.q[1, 3, 5] = was
        c.out[1, 3] = want[1, 3]
        c.check()


@every
@pytest.mark.parametrize("page", [16, 64])
def test_behind_the_length(most, page):
    """NaN codes behind an entry's last token, in its page and in pages behind."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, page, [71, 130, 255], [most, 1, most])
    want = c.run().clone()
    for b, t in enumerate(c.hc.lens):
        for p in range(t // page, c.hc.table.shape[1]):
            at = t - p * page if p == t // page else 0
            for name in ("k", "v"):
                c.hc.cache.t[name].view(torch.uint8)[int(c.hc.table[b, p]), :, at:] = 0x7f
    c.run()
    c.check()
    assert torch.equal(c.out, want)


@every
def test_many_entries(most):
    B = 70
    c = Case("bf16", "int8", 4, 1, 64, 16, [(37 * b) % 301 + 1 for b in range(B)], [min(m, (37 * b) % 301 + 1) for b, m in
                                                                                   enumerate(new_of(most, B))])
    c.most = most
    c.run()
    c.check()


@every
def test_entries_of_one_length(most):
    c = Case("fp16", "e4m3", 16, 4, 128, 64, [1500] * 6, [most] * 6, ragged=False)
    c.run()
    c.check()


@every
def test_rows_behind_the_last_entry(most):
    """Fewer rows than the call is told of: start's last one counts."""
    c = Case("fp16", "e4m3", 8, 2, 64, 16, [300, 90], [most, 1], tail=9)
    n, c.n = c.n, c.n + 7
    c.run()
    c.n = n
    c.check()


@every
def test_in_place_and_shared_pages(most):
    """Outputs over the queries; two entries that begin with the same pages."""
    torch = torch_cuda()
    c = Case("bf16", "e4m3", 8, 2, 128, 16, [1700, 420, 500], [most, most, most])
    c.hc.table[2, :10] = c.hc.table[1, :10]
    c.hc.cache.t["page_table"].copy_(device(c.hc.table))
    want = c.run().clone()
    c.check()
    q = c.q.clone()
    for _ in range(5):
        c.q.copy_(q)
        c.run(out=c.q)
        torch.cuda.synchronize()
        assert torch.equal(c.q[:c.n], want[:c.n])
        assert torch.equal(c.q[c.n:], q[c.n:])
    assert mkv.mkv_get_status() == 0


@every
def test_twice_the_same(most):
    torch = torch_cuda()
    c = Case("fp16", "int8", 8, 2, 128, 16, [5000, 420, 1500], new_of(most, 3))
    want = c.run().clone()
    for _ in range(5):
        c.out[:c.n].fill_(0)
        c.run()
        assert torch.equal(c.out, want)
    c.check()


@every
def test_far_offsets(most):
    """A pool, rows and outputs whose offsets pass 32 bits: bit for bit what the same bytes give close together."""
    torch = torch_cuda()
    c = Case("bf16", "e4m3", 8, 2, 128, 64, [300, 200], [most, 2])
    want = c.run()[:c.n].clone()
    per = 2 * 64 * 128
    far = (1 << 32) // per + 50                            # pages before the ones that are used
    t, ids = c.hc.cache.t, torch.arange(t_pages := c.hc.table.size, device="cuda", dtype=torch.int64) + far
    pools = {}
    for name in ("k", "v"):
        pools[name] = torch.empty((far + t_pages, 2, 64, 128), dtype=t[name].dtype, device="cuda")
        pools[name].view(torch.uint8)[far:] = t[name].view(torch.uint8)[device(c.hc.table.reshape(-1)).long()]
        pools[name + "_scale"] = torch.ones((far + t_pages, 2), device="cuda")
        pools[name + "_scale"][far:] = t[name + "_scale"][device(c.hc.table.reshape(-1)).long()]
    from paper_2609_07966_gb300 import caches
    cache = caches.wrap_paged_cache(c.cfg, ids.to(torch.int32).reshape(c.hc.table.shape), t["T_len"], pools["k"], pools["v"],
                                    pools["k_scale"], pools["v_scale"])
    stride = (1 << 31) // (c.n - 1) // 8 * 8 + 1024        # the last row lies past 2^32 bytes
    q, out = (torch.empty(stride * (c.n - 1) + 1024, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = lambda x: x.as_strided((c.n, 8, 128), (stride, 128, 1))
    rows(q).copy_(c.q[:c.n])
    mkv.mkv_paged_attention(c.cfg, q.data_ptr(), stride, c.start.data_ptr(), c.n, c.most, cache.c, out.data_ptr(), stride,
                            c.ws.data_ptr(), c.nws)
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == 0
    assert torch.equal(rows(out), want)


@every
def test_short_entries_beside_long_ones(most):
    """Some entries with hundreds of times the others' tokens: work is shared out in runs that hold several entries."""
    B = 20
    lens = [6000 if b in (3, 11) else most + 13 * b for b in range(B)]
    c = Case("bf16", "e4m3", 8, 2, 64, 16, lens, [most if b % 4 else max(1, most - b) for b in range(B)])
    c.run()
    c.check()


@every
def test_one_graph_for_all_lengths(most):
    """A call captured once, replayed as the entries' lengths change on the device (and with them how work is shared out)."""
    torch = torch_cuda()
    c = Case("fp16", "int8", 8, 2, 128, 32, [4000, 300, 2000], [most, most, 1], max_pages=126)
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=side):
        c.run(torch.cuda.current_stream().cuda_stream)
    for lens in ([4000, 300, 2000], [most, 90, 1], [0, 0, 0], [129, 4032, 700], [4032, 4032, 4032]):
        c.hc.lens = np.array(lens, dtype=np.int32)
        c.hc.cache.t["T_len"].copy_(device(c.hc.lens))
        c.out[:c.n].fill_(5)
        g.replay()
        c.check(what=f"{lens}")

"""Attention over 8-bit pages where few units' tiles are shared out among the CTAs (caches of 1152 tokens and more): what can go
wrong in pieces of a unit and in their join."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from paged_util import check_attention, device
from test_gpu_paged_attention import Case

pytestmark = pytest.mark.gpu

# most new tokens of an entry, times 4 heads a group: 120, 280 and 1200 query rows a key head
every = pytest.mark.parametrize("most", [30, 70, 300])


@every
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("D", [64, 128])
def test_missing_pages(most, page, D):
    """Single pages outside the pool, whole tiles of them (pieces that see nothing), the newest tokens' too; an entry without
    any gets NaN."""
    torch = torch_cuda()
    c = Case("bf16", "e4m3", 8, 2, D, page, [2850, 1300, 1471, 1290], [most, 1, most, most])
    t, pages = c.hc.cache.t["page_table"], c.hc.table.shape[1]
    gone = [np.zeros(pages, bool) for _ in range(4)]
    gone[0][[1, 700 // page]] = True
    gone[0][1024 // page:1664 // page] = True
    gone[2][:640 // page] = True
    gone[2][1471 // page - (0 if page == 128 else 3):] = True
    gone[3][:] = True
    for b in range(4):
        t[b, device(np.flatnonzero(gone[b]))] = -1 if b % 2 else 1 << 30
    c.run()
    c.check(flags=mkv.MKV_FLAG_BAD_INDEX, entries=(0, 1, 2), seen=lambda b, n: ~gone[b][np.arange(n) // page])
    assert torch.isnan(c.out[c.starts[3]:c.n]).all()


@every
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("x", [float("inf"), float("-inf"), float("nan")])
def test_queries_not_finite(most, D, x):
    """NaN in the row itself, whatever its pieces' maxima are; the others are right."""
    torch = torch_cuda()
    c = Case("bf16", "int8", 8, 2, D, 16, [2850, 1300], [most, most // 2])
    want, was = c.run().clone(), c.q[most // 2, 3, 5].clone()
    c.q[most // 2, 3, 5] = x
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[most // 2, 3]).all()
    c.q[most // 2, 3, 5] = was
    c.out[most // 2, 3] = want[most // 2, 3]
    c.check()


@every
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_all_infinite(most, sign):
    """Every score of a row plus or minus infinity: no weight is left, in any piece."""
    torch = torch_cuda()
    c = Case("fp16", "int8", 8, 2, 64, 64, [2850, 1300], [most, most // 2])
    c.hc.k[..., 7] = 9 * sign
    c.hc.cache.t["k"].copy_(device(c.hc.k))
    want, was = c.run().clone(), c.q[1, 4, 7].clone()
    c.check()
    c.q[1, 4, 7] = float("inf")
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[1, 4]).all()
    c.q[1, 4, 7] = was
    c.out[1, 4] = want[1, 4]
    c.check()


@every
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fmt,page", [("e4m3", 16), ("int8", 64)])
def test_scales_far_apart(most, D, fmt, page):
    """Pieces whose second maxima lie far from one another."""
    c = Case("bf16", fmt, 8, 2, D, page, [2850, 1300, 90], [most, most // 2, min(most, 90)], wild=30)
    c.run()
    c.check()


@every
@pytest.mark.parametrize("std,scale", [(2.0 ** 40, 2.0 ** -43), (2.0 ** -60, 2.0 ** 56)])
def test_large_and_small_queries(most, std, scale):
    c = Case("bf16", "e4m3", 8, 2, 64, 64, [2850, 1300], [most, most], std=std, scale=scale)
    c.run()
    c.check()


@every
@pytest.mark.parametrize("page", [16, 64])
def test_behind_the_length(most, page):
    """NaN codes behind an entry's last token, in its page and in pages behind."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, page, [2850, 1300, 1471], [most, 1, most])
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
def test_rows_before_the_first_position(most):
    """Entries of no tokens, one, and fewer than rows, beside one that is shared out."""
    torch = torch_cuda()
    c = Case("fp16", "e4m3", 8, 2, 128, 32, [0, 1, most - 1, 2850], [most] * 4)
    c.run()
    c.check()
    assert (c.out[:2 * most - 1] == 0).all() and (c.out[2 * most] == 0).all()


@every
def test_too_many_rows(most):
    """An entry with more rows than the call allows is left out; the others' pieces are joined."""
    torch = torch_cuda()
    c = Case("fp16", "int8", 8, 2, 64, 16, [1800, 1800, 1800], [most, most + 1, 1])
    c.most = most
    c.run()
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_BAD_INDEX
    assert (c.out[most:2 * most + 1] == 3).all()
    check_attention(c.hc, c.q, c.starts, c.out, c.dtype, entries=(0, 2))


@every
def test_far_offsets(most):
    """A pool whose offsets pass 32 bits: bit for bit what the same bytes give close together."""
    torch = torch_cuda()
    c = Case("bf16", "e4m3", 8, 2, 128, 64, [2850, 1300], [most, 2])
    want = c.run()[:c.n].clone()
    far = (1 << 32) // (2 * 64 * 128) + 50                 # pages before the ones that are used
    t, count = c.hc.cache.t, c.hc.table.size
    ids = torch.arange(count, device="cuda", dtype=torch.int64) + far
    at = device(c.hc.table.reshape(-1)).long()
    pools = {}
    for name in ("k", "v"):
        pools[name] = torch.empty((far + count, 2, 64, 128), dtype=t[name].dtype, device="cuda")
        pools[name].view(torch.uint8)[far:] = t[name].view(torch.uint8)[at]
        pools[name + "_scale"] = torch.ones((far + count, 2), device="cuda")
        pools[name + "_scale"][far:] = t[name + "_scale"][at]
    cache = caches.wrap_paged_cache(c.cfg, ids.to(torch.int32).reshape(c.hc.table.shape), t["T_len"], pools["k"], pools["v"],
                                    pools["k_scale"], pools["v_scale"])
    c.out[:c.n].fill_(0)
    mkv.mkv_paged_attention(c.cfg, c.q.data_ptr(), 0, c.start.data_ptr(), c.n, c.most, cache.c, c.out.data_ptr(), 0,
                            c.ws.data_ptr(), c.nws)
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == 0
    assert torch.equal(c.out[:c.n], want)


@every
def test_more_than_32_entries(most):
    """Lengths beyond a warp's lanes, most of them short, some shared out."""
    lens = [2850 if b in (0, 37) else 5 + 3 * b for b in range(40)]
    c = Case("bf16", "e4m3", 8, 2, 64, 16, lens, [most if b in (0, 37) else b % 3 for b in range(40)])
    c.run()
    c.check()

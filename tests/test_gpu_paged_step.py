"""The paged operators together, as a server runs them: prompts join the cache and are attended to, then steps of single and
drafted tokens, over several layers that share one workspace, eagerly and as one captured graph."""
import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import paged as P
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import SCORE, TINY, U, f64, randn, torch_dtype
from oracle.latent import attend_visible
from paged_util import FORMATS, KINDS, LAYOUTS, device, seeded

pytestmark = pytest.mark.gpu

LAYERS = 2


class Server:
    """LAYERS caches over one page table and one workspace, and the same caches' pages in the oracle."""

    def __init__(self, dtype, fmt, Hq, Hkv, D, page, B, pages, most_rows, layout="half"):
        torch = torch_cuda()
        self.rng = seeded("server", dtype, fmt, Hq, Hkv, D, page, B)
        self.dtype, self.fmt, self.page, self.B, self.Hq, self.Hkv, self.D, self.layout = dtype, fmt, page, B, Hq, Hkv, D, layout
        self.cfg = mkv.paged_config(KINDS[dtype], FORMATS[fmt], B, Hq, Hkv, D, page)
        self.rope = mkv.rope_config(D, layout=LAYOUTS[layout], scaling=mkv.MKV_ROPE_BANDS, theta=500000.0, factor=8.0, low=1.0,
                                    high=4.0, context=64)
        self.T = pages * page
        self.table = caches.rope_table(self.rope, self.T)
        num = B * pages + 2
        ids = self.rng.permutation(num)[:B * pages].reshape(B, pages).astype(np.int32)
        self.ids = ids
        self.caches = []
        for _ in range(LAYERS):
            c = caches.alloc_paged_cache(self.cfg, num, pages)
            c.t["page_table"].copy_(device(ids))
            self.caches.append(c)
        self.codes = [{x: (np.zeros((num, Hkv, page, D), np.int8 if fmt == "int8" else np.uint8), np.ones((num, Hkv), np.float32))
                       for x in "kv"} for _ in range(LAYERS)]
        self.lens = np.zeros(B, np.int64)
        self.ws, self.nws = caches.paged_workspace(self.cfg, most_rows * B, most_rows)
        for rows in (1, 2, 40, most_rows):
            b = mkv.mkv_paged_workspace_size(self.cfg, rows * B, rows)
            if b > self.nws:
                self.ws, self.nws = torch.zeros(b, dtype=torch.uint8, device="cuda"), b

    def inputs(self, n):
        return [randn(self.rng, (n, self.Hq + 2 * self.Hkv, self.D), self.dtype) for _ in range(LAYERS)]

    def step(self, qkv, start, n, most, outs):
        """One launch after another on the current stream; nothing is read back."""
        torch = torch_cuda()
        row = (self.Hq + 2 * self.Hkv) * self.D
        st = torch.cuda.current_stream().cuda_stream
        at = start.data_ptr() if start is not None else 0
        for layer in range(LAYERS):
            x, c = qkv[layer], self.caches[layer]
            k, v = x[:, self.Hq:], x[:, self.Hq + self.Hkv:]
            rows = mkv.paged_rows(n, start=at, q=x.data_ptr(), q_stride=row, q_out=outs[layer].data_ptr(), k=k.data_ptr(), k_stride=row,
                                  v=v.data_ptr(), v_stride=row)
            mkv.mkv_paged_append(self.cfg, self.rope, self.table.data_ptr(), self.T, rows, c.c, st)
            # (the rotated queries are read before the output takes their place)
            mkv.mkv_paged_attention(self.cfg, outs[layer].data_ptr(), 0, at, n, most, c.c, outs[layer].data_ptr(), 0,
                                    self.ws.data_ptr(), self.nws, st)

    def check(self, qkv, new, outs, what, lengths=True):
        torch = torch_cuda()
        torch.cuda.synchronize()
        assert mkv.mkv_get_status() == 0, what
        starts = np.concatenate([[0], np.cumsum(new)])
        G, Hq, Hkv, page = self.Hq // self.Hkv, self.Hq, self.Hkv, self.page
        pos = np.concatenate([t + np.arange(m) for t, m in zip(self.lens, new)])
        cs = self.table.cpu().numpy()[pos]
        for layer in range(LAYERS):
            x = qkv[layer].float().cpu().numpy()
            turned = P.rotate(x[:, :Hq + Hkv], cs, self.layout)
            q = f64(torch.from_numpy(turned[:, :Hq]).to(torch_dtype(self.dtype)))
            k, v = turned[:, Hq:], x[:, Hq + Hkv:]
            for b, m in enumerate(new):
                t = int(self.lens[b])
                for h in range(Hkv):
                    tokens = []
                    for name, y in (("k", k), ("v", v)):
                        codes, scales = self.codes[layer][name]
                        for p in range(t // page, (t + m - 1) // page + 1 if m else t // page):
                            i0, i1, pid = max(0, p * page - t), min(m, (p + 1) * page - t), self.ids[b, p]
                            scales[pid, h] = P.append_page(codes[pid, h], scales[pid, h], max(0, t - p * page),
                                                           y[starts[b] + i0:starts[b] + i1, h], self.fmt)
                        ids = self.ids[b, :-(-(t + m) // page)]
                        z = P.decode(codes[ids, h], self.fmt) * scales[ids, h].astype(np.float64)[:, None, None]
                        tokens.append(z.reshape(-1, self.D)[:t + m])
                    if m == 0:
                        continue
                    vis = np.arange(t + m)[None, :] <= (t + np.arange(m))[:, None]
                    rows = q[starts[b]:starts[b] + m, h * G:(h + 1) * G].reshape(m * G, -1)
                    ref, mag = attend_visible(rows, *tokens, np.repeat(vis, G, axis=0), self.D ** -0.5)
                    got = f64(outs[layer])[starts[b]:starts[b] + m, h * G:(h + 1) * G].reshape(m * G, -1)
                    # (tests/paged_util.py)
                    tol = (U["fp16"] + 2 * SCORE) * mag + U[self.dtype] * np.abs(ref) + (t + m) * 2.0 ** -31 * np.abs(tokens[1]).max() \
                        + TINY[self.dtype]
                    bad = ~(np.abs(got - ref) <= tol)
                    assert not bad.any(), f"{what} layer {layer} b{b} h{h}: {int(bad.sum())} of {bad.size} off, worst " \
                                          f"{np.abs(got - ref).max():.3e}"
        self.lens += np.asarray(new)
        for c in self.caches if lengths else ():
            assert c.t["T_len"].cpu().numpy().tolist() == self.lens.tolist(), what


@pytest.mark.parametrize("dtype,fmt,Hq,Hkv,D,page,layout", [("bf16", "e4m3", 8, 2, 128, 16, "half"), ("fp16", "int8", 4, 4, 64, 64, "pairs"),
                                                            ("bf16", "int8", 14, 2, 64, 32, "half")])
def test_prompts_then_steps(dtype, fmt, Hq, Hkv, D, page, layout):
    torch = torch_cuda()
    s = Server(dtype, fmt, Hq, Hkv, D, page, 3, 512 // page, 200, layout)
    for new in ([150, 40, 7], [1, 1, 1], [5, 1, 8], [0, 90, 33], [1, 1, 1], [2, 0, 1]):
        n = sum(new)
        qkv, outs = s.inputs(n), [torch.empty(n, Hq, D, dtype=torch_dtype(dtype), device="cuda") for _ in range(LAYERS)]
        start = device(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        s.step(qkv, start, n, max(new), outs)
        s.check(qkv, new, outs, f"{new}")


def test_captured_steps():
    """A step of every entry's next token, captured once and replayed on inputs that change: lengths live on the device."""
    torch = torch_cuda()
    s = Server("fp16", "e4m3", 8, 2, 128, 16, 4, 16, 1)
    n = 4
    qkv, outs = s.inputs(n), [torch.empty(n, 8, 128, dtype=torch.float16, device="cuda") for _ in range(LAYERS)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        s.step(qkv, None, n, 1, outs)
    for i in range(40):
        for x, y in zip(qkv, s.inputs(n)):
            x.copy_(y)
        graph.replay()
        s.check(qkv, [1] * n, outs, f"step {i}")


def test_two_streams():
    """Two servers' steps enqueued on two streams at once, and all of them checked afterwards."""
    torch = torch_cuda()
    servers = [Server("bf16", "int8", 8, 2, 64, 16, 2, 16, 60, layout) for layout in ("half", "pairs")]
    jobs = []
    for new in ([33, 60], [1, 1], [9, 4], [1, 0]):
        n = sum(new)
        start = device(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        for s in servers:
            jobs.append((s, s.inputs(n), start, n, new, [torch.empty(n, 8, 64, dtype=torch.bfloat16, device="cuda")
                                                         for _ in range(LAYERS)]))
    streams = {id(s): torch.cuda.Stream() for s in servers}
    torch.cuda.synchronize()
    for s, qkv, start, n, new, outs in jobs:
        with torch.cuda.stream(streams[id(s)]):
            s.step(qkv, start, n, max(new), outs)
    for s, qkv, start, n, new, outs in jobs:
        s.check(qkv, new, outs, f"{new}", lengths=False)
    for s in servers:
        assert all(c.t["T_len"].cpu().numpy().tolist() == s.lens.tolist() for c in s.caches)


@pytest.mark.parametrize("new", [[1, 3], [200, 90]])
def test_append_far_offsets(new):
    """Rows and a pool whose offsets pass 32 bits: bit for bit what the same call writes close together."""
    torch = torch_cuda()
    rng, Hq, Hkv, D, page, B = seeded("far", tuple(new)), 8, 2, 128, 64, 2
    cfg, rope = mkv.paged_config(mkv.MKV_BF16, mkv.MKV_I8, B, Hq, Hkv, D, page), mkv.rope_config(D)
    table, lens, most, n = caches.rope_table(rope, 512), [70, 0], 5, sum(new)
    qkv = randn(rng, (n, Hq + 2 * Hkv, D), "bf16")
    start = device(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    before = (1 << 32) // (Hkv * page * D) + 50
    got = []
    for first, stride in ((0, (Hq + 2 * Hkv) * D), (before, (1 << 31) // (n - 1) // 8 * 8 + (Hq + 2 * Hkv) * D)):
        pools = [torch.zeros((first + B * most, Hkv, page, D), dtype=torch.int8, device="cuda") for _ in range(2)]
        scales = [torch.ones((first + B * most, Hkv), device="cuda") for _ in range(2)]
        ids = (torch.arange(B * most, device="cuda") + first).to(torch.int32).reshape(B, most)
        c = caches.wrap_paged_cache(cfg, ids, device(np.array(lens, np.int32)), *pools, *scales)
        x, out = (torch.zeros(stride * (n - 1) + (Hq + 2 * Hkv) * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        x.as_strided(qkv.shape, (stride, D, 1)).copy_(qkv)
        rows = mkv.paged_rows(n, start=start.data_ptr(), q=x.data_ptr(), q_stride=stride, k=x[Hq * D:].data_ptr(), k_stride=stride,
                              v=x[(Hq + Hkv) * D:].data_ptr(), v_stride=stride, q_out=out.data_ptr(), q_out_stride=stride)
        mkv.mkv_paged_append(cfg, rope, table.data_ptr(), 512, rows, c.c)
        torch.cuda.synchronize()
        assert mkv.mkv_get_status() == 0
        got.append([y[first:].clone() for y in pools + scales] + [c.t["T_len"], out.as_strided((n, Hq, D), (stride, D, 1)).clone()])
    for y, z in zip(*got):
        assert torch.equal(y, z)


def test_rope_far_offsets():
    torch = torch_cuda()
    rng, n, heads, D = seeded("far rope"), 9, 5, 128
    cfg = mkv.rope_config(D)
    table, pos = caches.rope_table(cfg, 512), device(rng.integers(0, 512, n).astype(np.int32))
    src = randn(rng, (n, heads, D), "bf16")
    got = []
    for stride in (heads * D, (1 << 31) // (n - 1) + heads * D):
        x, out = (torch.zeros(stride * (n - 1) + heads * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        x.as_strided(src.shape, (stride, D, 1)).copy_(src)
        mkv.mkv_rope_apply(cfg, mkv.MKV_BF16, x.data_ptr(), stride, pos.data_ptr(), n, heads, table.data_ptr(), 512, 0, out.data_ptr(),
                           stride)
        got.append(out.as_strided(src.shape, (stride, D, 1)).clone())
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == 0 and torch.equal(*got)


@pytest.mark.parametrize("rows", [1, 9, 130])
def test_as_many_entries_as_there_may_be(rows):
    """4096 entries: their rows are appended (entries without any among them) and attended to; some of them are checked."""
    torch = torch_cuda()
    B, rng = 4096, seeded("many", rows)
    new = rng.integers(0, rows + 1, B) if rows < 100 else np.where(np.arange(B) % 64 == 5, rows, rng.integers(0, 3, B))
    new[:2] = rows, 0
    cfg = mkv.paged_config(mkv.MKV_F16, mkv.MKV_E4M3, B, 2, 1, 64, 16)
    held, pages, n = rng.integers(0, 20, B), 11, int(new.sum())
    c = caches.alloc_paged_cache(cfg, B * pages, pages)
    c.t["page_table"].copy_(torch.arange(B * pages, device="cuda").to(torch.int32).reshape(B, pages))
    qkv, q = randn(rng, (n + int(held.sum()), 4, 64), "fp16"), torch.empty(n, 2, 64, dtype=torch.float16, device="cuda")
    ws, nws = caches.paged_workspace(cfg, n, rows)

    def append(x, m):
        start = device(np.concatenate([[0], np.cumsum(m)]).astype(np.int32))
        mkv.mkv_paged_append(cfg, None, 0, 0, mkv.paged_rows(len(x), start=start.data_ptr(), k=x[:, 2:].data_ptr(), k_stride=256,
                                                             v=x[:, 3:].data_ptr(), v_stride=256), c.c)
        torch.cuda.synchronize()
        return start
    append(qkv[n:], held)
    start = append(qkv[:n], new)
    q.copy_(qkv[:n, :2])
    mkv.mkv_paged_attention(cfg, q.data_ptr(), 0, start.data_ptr(), n, rows, c.c, q.data_ptr(), 0, ws.data_ptr(), nws)
    torch.cuda.synchronize()
    assert mkv.mkv_get_status() == 0
    assert c.t["T_len"].cpu().numpy().tolist() == (held + new).tolist()
    first, before = np.concatenate([[0], np.cumsum(new)]), np.concatenate([[0], np.cumsum(held)]) + n
    host = f64(qkv)
    for b in [0, 5, 69, 4095] + list(rng.choice(B, 60)):
        m, t = int(new[b]), int(held[b] + new[b])
        tokens = []
        for i, name in ((2, "k"), (3, "v")):
            x = np.concatenate([host[before[b]:before[b + 1], i], host[first[b]:first[b + 1], i]])
            ids = slice(b * pages, b * pages + -(-t // 16))
            z = P.decode(c.t[name].view(torch.uint8)[ids, 0].cpu().numpy(), "e4m3") * \
                f64(c.t[name + "_scale"][ids, 0])[:, None, None]
            z = z.reshape(-1, 64)[:t]
            # a code is off by half a step, 2^-4 of the value; where its page's scale grew, what fell below the normal range was
            # rounded again, by half of the least step, 2^-10 of a scale that is at most 2 / 448 of the page's largest value
            assert (np.abs(z - x) <= 2.0 ** -3 * np.abs(x) + 2.0 ** -9 * np.abs(x).max(initial=0.0)).all(), b
            tokens.append(z)
        if m:
            vis = np.arange(t)[None, :] <= (t - m + np.arange(m))[:, None]
            ref, mag = attend_visible(host[first[b]:first[b + 1], :2].reshape(2 * m, 64), *tokens, np.repeat(vis, 2, axis=0), 0.125)
            got = f64(q)[first[b]:first[b + 1]].reshape(2 * m, 64)
            tol = (U["fp16"] + 2 * SCORE) * mag + U["fp16"] * np.abs(ref) + t * 2.0 ** -31 * np.abs(tokens[1]).max() + TINY["fp16"]
            assert (np.abs(got - ref) <= tol).all(), b

"""One call each of the tree and latent attention operators on given tensors, as the edge tests make them."""
import paper_2609_07966_gb300 as mkv
from paper_2609_07966_gb300 import caches

from gpu_util import torch_cuda
from latent_util import to_mask

KINDS = {"fp16": mkv.MKV_F16, "bf16": mkv.MKV_BF16}


def _lens(lens):
    import torch
    return torch.tensor(lens, dtype=torch.int32, device="cuda")


def _workspace(pair):
    """A workspace whose contents past its counters are junk."""
    ws, nbytes = pair
    ws.fill_(255)
    ws[:16384] = 0
    return ws, nbytes


def padded(x, dim, size, junk):
    """x with `size` entries along dim, those past its own holding `junk`."""
    import torch
    shape = list(x.shape)
    shape[dim] = size
    out = torch.full(shape, junk, dtype=x.dtype, device=x.device)
    out.narrow(dim, 0, x.shape[dim]).copy_(x)
    return out


def tree_plan(q, k, v, lens):
    """What a program keeps for tree attention of q [B][n][Hq][D] over k, v [B][Hkv][T_cap][D]."""
    torch_cuda()
    B, n, Hq, D = q.shape
    cfg = mkv.config(mkv.MKV_FP16, B, Hq, k.shape[1], D)
    return cfg, caches.wrap_cache(cfg, _lens(lens), k, v), _workspace(caches.tree_workspace(cfg, k.shape[2], n))


def tree_call(plan, q, kt, vt, mask, out, stream=None):
    cfg, cache, (ws, nws) = plan
    mkv.mkv_tree_attention(cfg, q.data_ptr(), cache.c, kt.data_ptr(), vt.data_ptr(), mask.data_ptr(), q.shape[1],
                           out.data_ptr(), ws.data_ptr(), nws, stream)


def tree(q, k, v, lens, kt, vt, masks):
    import torch
    out, mask, plan = torch.full_like(q, 3.0), to_mask(masks), tree_plan(q, k, v, lens)
    torch.cuda.synchronize()
    tree_call(plan, q, kt, vt, mask, out)
    assert mkv.mkv_get_status() == 0
    return out


def latent_plan(dtype, q, rows, lens):
    """What a program keeps for latent attention of q [B][n][H][rank + 64] over rows [B][T_cap][rank + 64]."""
    torch_cuda()
    B, n, H, row = q.shape
    cfg = mkv.latent_config(KINDS[dtype], B, H, rank=row - 64)
    return (cfg, caches.wrap_latent_cache(cfg, _lens(lens), rows),
            _workspace(caches.latent_workspace(cfg, rows.shape[1], n)))


def latent_call(plan, q, new, mask, out, stream=None):
    cfg, cache, (ws, nws) = plan
    mkv.mkv_latent_attention(cfg, q.data_ptr(), cache.c, 0 if new is None else new.data_ptr(),
                             0 if new is None else mask.data_ptr(), q.shape[1], out.data_ptr(), ws.data_ptr(), nws,
                             stream)


def latent(dtype, q, rows, lens, new=None, masks=None):
    import torch
    out = torch.full(q.shape[:3] + (q.shape[3] - 64,), 3.0, dtype=q.dtype, device="cuda")
    mask, plan = None if masks is None else to_mask(masks), latent_plan(dtype, q, rows, lens)
    torch.cuda.synchronize()
    latent_call(plan, q, new, mask, out)
    assert mkv.mkv_get_status() == 0
    return out


def prefill(dtype, q, kv, rope, lens, rank=256):
    """Queries [B][n][H][nope + 64] over kv [B][H][T][nope + v] and the rotated keys rope [B][T][64]."""
    import torch
    torch_cuda()
    B, n, H, dk = q.shape
    T, vdim = kv.shape[2], kv.shape[3] - (dk - 64)
    cfg = mkv.latent_config(KINDS[dtype], B, H, rank=rank, nope_dim=dk - 64, v_dim=vdim)
    rows = torch.zeros((B, T, rank + 64), dtype=q.dtype, device="cuda")
    rows[..., rank:] = rope
    cache = caches.wrap_latent_cache(cfg, _lens(lens), rows)
    out = torch.full((B, n, H, vdim), 3.0, dtype=q.dtype, device="cuda")
    torch.cuda.synchronize()
    mkv.mkv_latent_prefill(cfg, q.data_ptr(), kv.data_ptr(), T, cache.c, 0, n, out.data_ptr())
    assert mkv.mkv_get_status() == 0
    return out

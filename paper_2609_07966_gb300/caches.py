"""Device-memory plumbing for libmkv: caches, calibration tables, workspace.

PyTorch only allocates here (torch tensors own the memory); the returned
objects carry the ctypes structs of include/mkv.h pointing into them.
"""
from __future__ import annotations

import dataclasses

from . import (MKV_BF16, MKV_E4M3, MKV_FP16, MKV_H2O, MKV_KVQUANT, MKV_ROCKET, mkv_cache, mkv_latent_cache,
               mkv_latent_workspace_size, mkv_paged_cache, mkv_paged_workspace_size, mkv_quant_params,
               mkv_rope_scaled_table, mkv_tree_workspace_size, mkv_workspace_size, n_value_outliers)


@dataclasses.dataclass
class Cache:
    """One layer's cache: torch tensors plus the mkv_cache struct over them."""
    cfg: object
    T_cap: int
    t: dict
    c: mkv_cache


def _ptr(x):
    return 0 if x is None else x.data_ptr()


def alloc_cache(cfg, T_cap: int, device="cuda", k_out_cap: int | None = None) -> Cache:
    """Zeroed cache of T_cap slots for cfg.method (T_len = 0, H2O slots empty)."""
    import torch
    B, Hkv, D = cfg.B, cfg.Hkv, cfg.D
    t = {"T_len": torch.zeros(B, dtype=torch.int32, device=device)}
    if cfg.method in (MKV_FP16, MKV_H2O, MKV_ROCKET):
        t["k"] = torch.zeros((B, Hkv, T_cap, D), dtype=torch.float16, device=device)
        t["v"] = torch.zeros((B, Hkv, T_cap, D), dtype=torch.float16, device=device)
    if cfg.method == MKV_H2O:
        t["pos"] = torch.full((B, Hkv, T_cap), -1, dtype=torch.int32, device=device)
        t["acc"] = torch.zeros((B, Hkv, T_cap), dtype=torch.float32, device=device)
        t["slot"] = torch.zeros((B, Hkv), dtype=torch.int32, device=device)
    if cfg.method == MKV_ROCKET:
        npg = T_cap // 16
        t["kmin"] = torch.zeros((B, Hkv, D, npg), dtype=torch.float16, device=device)
        t["kmax"] = torch.zeros((B, Hkv, D, npg), dtype=torch.float16, device=device)
    if cfg.method == MKV_KVQUANT:
        row = D * cfg.bits // 8
        nv = n_value_outliers(D, cfg.outlier_frac)
        if k_out_cap is None:   # 4x the nominal outlier rate (data beyond the calibration range)
            k_out_cap = int(T_cap * D * min(1.0, max(cfg.outlier_frac, 1e-6) * 4)) + 1024
        t["k_codes"] = torch.zeros((B, Hkv, T_cap, row), dtype=torch.uint8, device=device)
        t["v_codes"] = torch.zeros((B, Hkv, T_cap, row), dtype=torch.uint8, device=device)
        t["v_params"] = torch.zeros((B, Hkv, T_cap, 2), dtype=torch.float32, device=device)
        t["v_out"] = torch.zeros((B, Hkv, T_cap, max(nv, 1)), dtype=torch.int32, device=device)
        t["k_out_off"] = torch.zeros((B, Hkv, T_cap + 1), dtype=torch.int32, device=device)
        t["k_out"] = torch.zeros((B, Hkv, k_out_cap), dtype=torch.int32, device=device)
    c = mkv_cache()
    c.T_cap = T_cap
    for name, _ in mkv_cache._fields_:
        if name in t:
            setattr(c, name, _ptr(t[name]))
    c.k_out_cap = t["k_out"].shape[-1] if "k_out" in t else 0
    return Cache(cfg, T_cap, t, c)


@dataclasses.dataclass
class QuantParams:
    t: dict
    c: mkv_quant_params


def alloc_quant_params(cfg, rope_len: int, device="cuda") -> QuantParams:
    """Calibration tables of one layer (zeros) and a rope table of rope_len rows."""
    import torch
    Hkv, D, K = cfg.Hkv, cfg.D, 1 << cfg.bits
    t = {
        "t_lo": torch.zeros((Hkv, D), dtype=torch.float32, device=device),
        "t_hi": torch.zeros((Hkv, D), dtype=torch.float32, device=device),
        "k_lo": torch.zeros((Hkv, D), dtype=torch.float32, device=device),
        "k_scale": torch.zeros((Hkv, D), dtype=torch.float32, device=device),
        "k_cb": torch.zeros((Hkv, D, K), dtype=torch.float16, device=device),
        "v_cb": torch.zeros((Hkv, D, K), dtype=torch.float16, device=device),
        "k_dq": torch.zeros((Hkv, D, K), dtype=torch.float32, device=device),
        "v_tbl": torch.zeros((Hkv, D, K), dtype=torch.float16, device=device),
        "rope": torch.zeros((rope_len, D // 2, 2), dtype=torch.float32, device=device),
    }
    c = mkv_quant_params()
    for name, _ in mkv_quant_params._fields_:
        if name in t:
            setattr(c, name, _ptr(t[name]))
    c.rope_len = rope_len
    return QuantParams(t, c)


def workspace(cfg, T_cap: int, device="cuda"):
    """(tensor, nbytes) of the workspace mkv_workspace_size asks for, zero-filled
    (its leading counters must start at zero; the library keeps them zero)."""
    import torch
    n = mkv_workspace_size(cfg, T_cap)
    return torch.zeros(n, dtype=torch.uint8, device=device), n


def _check(name, t, dtype, shape, device):
    """ValueError unless t is a contiguous tensor of the type, of the shape (at least as many entries: its first
    dimension) and on the device: the kernels get its address alone."""
    want = f"{name} must be contiguous {dtype} of shape {list(shape)} (or more entries) on {device}"
    if t.dtype != dtype or t.device != device or t.dim() != len(shape) or not t.is_contiguous() or \
            t.shape[0] < shape[0] or tuple(t.shape[1:]) != tuple(shape[1:]):
        raise ValueError(f"{want}, not {t.dtype} of shape {list(t.shape)}, strides {list(t.stride())} on {t.device}")


def wrap_cache(cfg, T_len, k, v) -> Cache:
    """An FP16 cache over tensors the caller already has: k, v fp16 [B][Hkv][T_cap][D], T_len int32 [B], all
    contiguous and on one device; ValueError otherwise."""
    import torch
    shape = (cfg.B, cfg.Hkv, k.shape[2] if k.dim() == 4 else 0, cfg.D)
    _check("k", k, torch.float16, shape, k.device)
    _check("v", v, torch.float16, shape, k.device)
    _check("T_len", T_len, torch.int32, (cfg.B,), k.device)
    c = mkv_cache()
    c.T_cap, c.T_len, c.k, c.v = k.shape[2], _ptr(T_len), _ptr(k), _ptr(v)
    return Cache(cfg, k.shape[2], {"T_len": T_len, "k": k, "v": v}, c)


def tree_workspace(cfg, T_cap: int, n: int, device="cuda"):
    """(tensor, nbytes) of the workspace of mkv_tree_attention for n drafted tokens, zero-filled."""
    import torch
    b = mkv_tree_workspace_size(cfg, T_cap, n)
    return torch.zeros(b, dtype=torch.uint8, device=device), b


@dataclasses.dataclass
class LatentCache:
    """One layer's latent cache: torch tensors plus the mkv_latent_cache struct over them."""
    cfg: object
    T_cap: int
    t: dict
    c: mkv_latent_cache


def latent_dtype(cfg):
    import torch
    return torch.bfloat16 if cfg.dtype == MKV_BF16 else torch.float16


def wrap_latent_cache(cfg, T_len, rows) -> LatentCache:
    """A latent cache over tensors the caller already has: rows [B][T_cap][rank + rope_dim] of the configuration's type,
    T_len int32 [B], contiguous and on one device; ValueError otherwise."""
    import torch
    _check("rows", rows, latent_dtype(cfg), (cfg.B, rows.shape[1] if rows.dim() == 3 else 0, cfg.rank + cfg.rope_dim),
           rows.device)
    _check("T_len", T_len, torch.int32, (cfg.B,), rows.device)
    return LatentCache(cfg, rows.shape[1], {"T_len": T_len, "rows": rows},
                       mkv_latent_cache(rows.shape[1], _ptr(T_len), _ptr(rows)))


def alloc_latent_cache(cfg, T_cap: int, device="cuda") -> LatentCache:
    """Zeroed latent cache of T_cap slots (T_len = 0)."""
    import torch
    return wrap_latent_cache(cfg, torch.zeros(cfg.B, dtype=torch.int32, device=device),
                             torch.zeros((cfg.B, T_cap, cfg.rank + cfg.rope_dim), dtype=latent_dtype(cfg),
                                         device=device))


def latent_workspace(cfg, T_cap: int, n: int, device="cuda"):
    """(tensor, nbytes) of the workspace of mkv_latent_attention for n tokens per entry, zero-filled."""
    import torch
    b = mkv_latent_workspace_size(cfg, T_cap, n)
    return torch.zeros(b, dtype=torch.uint8, device=device), b


def rope_table(cfg, T_max: int, device="cuda", stream=None):
    """fp32 [T_max][rot_dim / 2][2]: the table of mkv_rope_scaled_table, filled on the device's current stream."""
    import torch
    t = torch.empty((T_max, cfg.rot_dim // 2, 2), dtype=torch.float32, device=device)
    with torch.cuda.device(t.device):
        mkv_rope_scaled_table(cfg, T_max, _ptr(t), stream)
    return t


@dataclasses.dataclass
class PagedCache:
    """One layer's 8-bit pages: torch tensors plus the mkv_paged_cache struct over them."""
    cfg: object
    t: dict
    c: mkv_paged_cache


def code_dtype(cfg):
    import torch
    return torch.float8_e4m3fn if cfg.format == MKV_E4M3 else torch.int8


def wrap_paged_cache(cfg, page_table, T_len, k, v, k_scale, v_scale, tickets=None) -> PagedCache:
    """A paged cache over tensors the caller already has: k, v [num_pages][Hkv][page_size][D] of code_dtype(cfg), k_scale,
    v_scale fp32 [num_pages][Hkv], page_table int32 [B][max_pages], T_len int32 [B], all contiguous and on one device;
    ValueError otherwise.  tickets int32 [B] zeros (allocated unless given)."""
    import torch
    num = k.shape[0] if k.dim() == 4 else 0
    shape = (num, cfg.Hkv, cfg.page_size, cfg.D)
    _check("k", k, code_dtype(cfg), shape, k.device)
    _check("v", v, code_dtype(cfg), shape, k.device)
    _check("k_scale", k_scale, torch.float32, (num, cfg.Hkv), k.device)
    _check("v_scale", v_scale, torch.float32, (num, cfg.Hkv), k.device)
    _check("page_table", page_table, torch.int32, (cfg.B, page_table.shape[1] if page_table.dim() == 2 else 0), k.device)
    _check("T_len", T_len, torch.int32, (cfg.B,), k.device)
    if tickets is None:
        tickets = torch.zeros(cfg.B, dtype=torch.int32, device=k.device)
    _check("tickets", tickets, torch.int32, (cfg.B,), k.device)
    t = {"page_table": page_table, "T_len": T_len, "tickets": tickets, "k": k, "v": v, "k_scale": k_scale,
         "v_scale": v_scale}
    return PagedCache(cfg, t, mkv_paged_cache(num, page_table.shape[1], **{x: _ptr(y) for x, y in t.items()}))


def alloc_paged_cache(cfg, num_pages: int, max_pages: int, device="cuda") -> PagedCache:
    """Zeroed pool of num_pages pages, empty entries, and a page table that names no page (-1) yet."""
    import torch
    shape = (num_pages, cfg.Hkv, cfg.page_size, cfg.D)
    k, v = (torch.zeros(shape, dtype=torch.int8, device=device).view(code_dtype(cfg)) for _ in range(2))
    ks, vs = (torch.ones(shape[:2], dtype=torch.float32, device=device) for _ in range(2))
    return wrap_paged_cache(cfg, torch.full((cfg.B, max_pages), -1, dtype=torch.int32, device=device),
                            torch.zeros(cfg.B, dtype=torch.int32, device=device), k, v, ks, vs)


def paged_workspace(cfg, n: int, max_rows: int, device="cuda"):
    """(tensor, nbytes) of the workspace of mkv_paged_attention for n rows, at most max_rows an entry, zero-filled."""
    import torch
    b = mkv_paged_workspace_size(cfg, n, max_rows)
    return torch.zeros(b, dtype=torch.uint8, device=device), b

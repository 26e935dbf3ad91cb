"""Caches over a caller's own tensors: what the kernels would read wrongly is refused before a pointer is taken (CPU)."""
import pytest

import paper_2609_07966_gb300 as mkv
from paper_2609_07966_gb300 import caches

torch = pytest.importorskip("torch")

B, HKV, T, D = 2, 3, 32, 64


def _fp16(T_len=None, k=None, v=None):
    cfg = mkv.config(mkv.MKV_FP16, B, 6, HKV, D)
    full = lambda: torch.zeros(B, HKV, T, D, dtype=torch.float16)      # noqa: E731
    return caches.wrap_cache(cfg, torch.zeros(B, dtype=torch.int32) if T_len is None else T_len,
                             full() if k is None else k, full() if v is None else v)


def _latent(T_len=None, rows=None, dtype=mkv.MKV_BF16):
    cfg = mkv.latent_config(dtype, B, 4, rank=256)
    return caches.wrap_latent_cache(cfg, torch.zeros(B, dtype=torch.int32) if T_len is None else T_len,
                                    torch.zeros(B, T, 320, dtype=torch.bfloat16) if rows is None else rows)


def test_fitting_tensors_are_taken_as_they_are():
    k = torch.zeros(B, HKV, T, D, dtype=torch.float16)
    c = _fp16(k=k)
    assert c.c.k == k.data_ptr() and c.T_cap == c.c.T_cap == T and c.t["k"] is k
    # a cache with room for more entries than the call has
    _fp16(T_len=torch.zeros(5, dtype=torch.int32), k=k.repeat(2, 1, 1, 1), v=k.repeat(2, 1, 1, 1))
    rows = torch.zeros(B + 1, T, 320, dtype=torch.bfloat16)
    c = _latent(rows=rows)
    assert c.c.rows == rows.data_ptr() and c.T_cap == c.c.T_cap == T
    assert caches.alloc_latent_cache(c.cfg, 7, device="cpu").T_cap == 7


@pytest.mark.parametrize("what,bad", [
    ("k", lambda: torch.zeros(B, HKV, T, D)),                                              # fp32
    ("v", lambda: torch.zeros(B, HKV, T, D, dtype=torch.bfloat16)),
    ("k", lambda: torch.zeros(B, HKV, T, D // 2, dtype=torch.float16)),                    # narrower rows
    ("k", lambda: torch.zeros(B, HKV + 1, T, D, dtype=torch.float16)),
    ("v", lambda: torch.zeros(B, HKV, T - 1, D, dtype=torch.float16)),                     # shorter than k
    ("v", lambda: torch.zeros(B - 1, HKV, T, D, dtype=torch.float16)),
    ("k", lambda: torch.zeros(B * HKV * T, D, dtype=torch.float16)),
    ("k", lambda: torch.zeros(B, T, HKV, D, dtype=torch.float16).transpose(1, 2)),         # token-major
    ("k", lambda: torch.zeros(B, HKV, 2 * T, D, dtype=torch.float16)[:, :, :T]),           # a slice of a longer one
    ("v", lambda: torch.zeros(B, HKV, T, D, dtype=torch.float16, device="meta")),
    ("T_len", lambda: torch.zeros(B, dtype=torch.int64)),
    ("T_len", lambda: torch.zeros(B - 1, dtype=torch.int32)),
    ("T_len", lambda: torch.zeros(B, 1, dtype=torch.int32)),
    ("T_len", lambda: torch.zeros(2 * B, dtype=torch.int32)[::2]),
    ("T_len", lambda: torch.zeros(B, dtype=torch.int32, device="meta")),
])
def test_fp16_refusals(what, bad):
    with pytest.raises(ValueError, match=what):
        _fp16(**{what: bad()})


@pytest.mark.parametrize("what,bad", [
    ("rows", lambda: torch.zeros(B, T, 320, dtype=torch.float16)),                         # the other 16-bit type
    ("rows", lambda: torch.zeros(B, T, 576, dtype=torch.bfloat16)),                        # another rank
    ("rows", lambda: torch.zeros(B - 1, T, 320, dtype=torch.bfloat16)),
    ("rows", lambda: torch.zeros(B * T, 320, dtype=torch.bfloat16)),
    ("rows", lambda: torch.zeros(T, B, 320, dtype=torch.bfloat16).transpose(0, 1)),
    ("rows", lambda: torch.zeros(B, T, 384, dtype=torch.bfloat16)[..., :320]),
    ("T_len", lambda: torch.zeros(B, dtype=torch.int64)),
    ("T_len", lambda: torch.zeros(B - 1, dtype=torch.int32)),
    ("T_len", lambda: torch.zeros(B, dtype=torch.int32, device="meta")),
])
def test_latent_refusals(what, bad):
    with pytest.raises(ValueError, match=what):
        _latent(**{what: bad()})

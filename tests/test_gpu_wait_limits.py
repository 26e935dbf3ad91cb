"""The bounded waits of the tree and latent kernels run out (on a barrier that nothing arrives on): the CTA waits for its
copies and products under way, reports, and leaves the context usable."""
import time

import numpy as np
import pytest

import paper_2609_07966_gb300 as mkv
from oracle import latent as L

import tree_latent_calls as calls
from gpu_util import torch_cuda
from latent_util import check_attention, f64, randn

pytestmark = pytest.mark.gpu


def test_role_waits_run_out_and_the_next_calls_are_right():
    torch_cuda()
    assert mkv.mkv_get_status() == 0
    mkv.mkv_wait_timeout_selftest(1)                     # (code loaded)
    mkv.mkv_get_status()
    t0 = time.perf_counter()
    mkv.mkv_wait_timeout_selftest(30)
    assert mkv.mkv_get_status() == mkv.MKV_FLAG_WAIT_TIMEOUT
    waited = time.perf_counter() - t0
    # two CTAs one after the other, 30 ms each; a copy or a product that the second one could not see the end of would
    # hold it for a second
    assert 0.055 < waited < 0.5, waited
    assert mkv.mkv_get_status() == 0
    rng = np.random.default_rng(1)
    q, kv, rope = (randn(rng, s, "fp16") for s in ((1, 130, 2, 192), (1, 2, 130, 256), (1, 130, 64)))
    out = calls.prefill("fp16", q, kv, rope, [130])
    for h in range(2):
        keys = np.concatenate([f64(kv[0, h, :, :128]), f64(rope[0])], 1)
        ref, mag = L.attend_visible(f64(q[0, :, h]), keys, f64(kv[0, h, :, 128:]), L.causal_visible(130, 130, 130),
                                    192 ** -0.5)
        check_attention(out[0, :, h], ref, mag, "fp16", f"h{h}")
    q, rows = randn(rng, (1, 1, 8, 320), "bf16"), randn(rng, (1, 200, 320), "bf16")
    ref, mag = L.attend_visible(f64(q).reshape(8, -1), f64(rows[0]), f64(rows[0, :, :256]), np.ones((8, 200), bool),
                                192 ** -0.5)
    check_attention(calls.latent("bf16", q, rows, [200]).reshape(8, 256), ref, mag, "bf16")

"""What reading the status word costs a caller."""
import time

import pytest

import paper_2609_07966_gb300 as mkv

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu


def _best(f, n=60):
    f()
    times = []
    for _ in range(n):
        t = time.perf_counter()
        f()
        times.append(time.perf_counter() - t)
    return min(times)


def test_status_costs_a_few_round_trips_at_most():
    """One word a unit, but not one round trip a unit: no more than six of them, the number that the library's first six
    units took, with a round trip taken as a word copied from the device, one copied to it, and a synchronisation."""
    torch = torch_cuda()
    word, host = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32)
    stream = torch.cuda.current_stream()

    def trip():
        host.copy_(word)
        word.copy_(host)
        stream.synchronize()
    trip_s, status_s = _best(trip), _best(mkv.mkv_get_status)
    assert status_s <= 6 * trip_s, f"status {status_s * 1e6:.1f} us, a round trip {trip_s * 1e6:.1f} us"

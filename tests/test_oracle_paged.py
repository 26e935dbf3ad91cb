"""The oracle of the rotary and paged operators, pinned by closed forms and torch's own conversions."""
import numpy as np
import pytest

from oracle import paged as P
from oracle import rope


def test_plain_half_rotation_is_the_other_oracles():
    x = np.random.default_rng(0).standard_normal((5, 3, 64))
    cs = P.table(np.arange(5) + 7, P.frequencies(64, 10000.0))
    want = rope.apply(x.transpose(1, 0, 2), np.arange(5) + 7, 10000.0).transpose(1, 0, 2)
    assert np.allclose(P.rotate(x, cs, "half"), want, atol=1e-12)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotations_compose_and_keep_lengths(layout):
    x = np.random.default_rng(1).standard_normal((4, 2, 40))
    f = P.frequencies(24)
    at = lambda p: P.table(np.full(4, p), f)
    y = P.rotate(P.rotate(x, at(3), layout), at(5), layout)
    assert np.allclose(y, P.rotate(x, at(8), layout))
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 24:], x[..., 24:])


def test_scaled_frequencies():
    plain = P.frequencies(128, 500000.0)
    assert np.allclose(P.frequencies(128, 500000.0, "linear", 4.0), plain / 4)
    for kind, low, high in (("bands", 1.0, 4.0), ("ramp", 1.0, 32.0)):
        f = P.frequencies(128, 500000.0, kind, 8.0, low, high, 8192)
        turns = 8192 * plain / (2 * np.pi)
        ratio = f / plain
        assert np.all(np.diff(ratio) <= 1e-12) and np.allclose(ratio[turns > high * 1.5], 1)
        assert np.allclose(ratio[turns < low / 1.5], 1 / 8)
        assert ((ratio > 1 / 8 + 1e-6) & (ratio < 1 - 1e-6)).any()


def test_codes_are_torchs():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.standard_normal(5000) * 2.0 ** rng.integers(-14, 9, 5000), P.E4M3[:127],
                        (P.E4M3[:126] + P.E4M3[1:127]) / 2, -P.E4M3[:127]]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    t = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(P.encode(x, "e4m3"), t.view(torch.uint8).numpy())
    back = P.decode(t.view(torch.uint8).numpy(), "e4m3")
    assert np.array_equal(back, t.float().numpy().astype(np.float64))
    assert P.encode(np.array([1e9, -np.inf, np.nan, 0.5, 1.5, -2.5], np.float32), "int8").tolist() == [127, -127, 0, 0, 2, -2]
    assert P.decode(P.encode(np.array([1e9, -np.inf, np.nan], np.float32), "e4m3"), "e4m3").tolist() == [448, -448, 0]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_least_scales(fmt):
    top = P.TOP[fmt]
    for e in (-100, -20, 0, 7, 120):
        assert P.least_scale(np.float32(top * 2.0 ** e), fmt) == 2.0 ** e
    assert P.least_scale(np.nextafter(np.float32(top), np.float32(1e9)), fmt) == 2.0
    assert P.least_scale(0.0, fmt) == 2.0 ** -100 and P.least_scale(3.4e38, "int8") == 2.0 ** 120


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_pages_keep_their_tokens_values(fmt):
    rng = np.random.default_rng(3)
    codes = P.encode(rng.standard_normal((16, 64)).astype(np.float32) * 30, fmt)
    was = P.decode(codes, fmt)[:10] * 0.25
    now = P.append_page(codes, np.float32(0.25), 10, rng.standard_normal((3, 64)).astype(np.float32) * 300, fmt)
    assert now > 0.25 and np.abs(P.decode(codes, fmt)[:10] * now - was).max() <= (now / 2 if fmt == "int8" else 2.0 ** -4 * np.abs(was).max())
    kept = codes.copy()
    assert P.append_page(codes, now, 13, np.zeros((1, 64), np.float32), fmt) == now and np.array_equal(codes[:13], kept[:13])

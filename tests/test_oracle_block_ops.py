"""The 64-bit references of the norm, the 8-bit products and the filtered sampling against what is known of them."""
import math

import numpy as np
import pytest

from oracle import block_ops as B


def test_norm_known():
    y, r = B.rms_norm(np.array([[3.0, 4.0]]), eps=0.0)
    assert np.allclose(r, 1 / math.sqrt(12.5)) and np.allclose((y * y).mean(), 1.0)
    y, _ = B.rms_norm(np.zeros((1, 5)), eps=1e-5)
    assert (y == 0).all()


@pytest.mark.parametrize("weighted", [True, False])
def test_norm_gradient_by_differences(weighted):
    g = np.random.default_rng(0)
    h, dy, dh = g.normal(size=(3, 7)), g.normal(size=(3, 7)), g.normal(size=(3, 7))
    w = g.normal(size=7) if weighted else None
    d, dw = B.rms_norm_grad(dy, h, B.rms_norm(h, w)[1], w, dh)

    def loss(h, w):
        return (dy * B.rms_norm(h, w)[0]).sum() + (dh * h).sum()
    for i in range(3):
        for k in range(7):
            e = np.zeros_like(h)
            e[i, k] = 1e-5
            assert abs((loss(h + e, w) - loss(h - e, w)) / 2e-5 - d[i, k]) < 1e-8
    for k in range(7 if weighted else 0):
        e = np.zeros(7)
        e[k] = 1e-5
        assert abs((loss(h, w + e) - loss(h, w - e)) / 2e-5 - dw[k]) < 1e-8


def test_e4m3_values():
    v = B.E4M3
    assert v[0x7e] == 448 and math.isnan(v[0x7f]) and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1 and v[0xb8] == -1
    codes = np.array([c for c in range(256) if not math.isnan(v[c])], np.uint8)
    assert (B.to_e4m3(v[codes]) == codes).all()


def test_e4m3_rounds_to_even():
    # between 16 and 18 lies 17, between 18 and 20 lies 19: both go to the even mantissa
    assert B.E4M3[B.to_e4m3([17.0, 19.0, 17.01, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 449.0])].tolist() == [
        16, 20, 18, -16, 0, 2 * 2.0 ** -9, 448]


@pytest.mark.parametrize("tile", [True, False])
def test_quantize_reaches_448(tile):
    x = np.random.default_rng(1).normal(size=(150, 200)).astype(np.float32)
    q, s = B.quantize(x, tile)
    assert s.shape == ((2, 2) if tile else (150, 2))
    back = B.E4M3[q] * B.widen(s, 150, 200, tile)
    assert (B.block_tops(np.abs(B.E4M3[q]), tile) == 448).all()
    assert (np.abs(back - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * B.widen(s, 150, 200, tile)).all()


def test_sample_filters():
    l, one = np.log([0.4, 0.1, 0.3, 0.2]), np.ones(4)
    assert B.sample(l, one)[:2] == (0, pytest.approx(0.4))
    assert B.sample(l, [9, 9, 1e-3, 1e-6], top_k=2)[:2] == (2, pytest.approx(3 / 7))
    assert B.sample(l, [9, 9, 9, 1e-6], top_p=0.75)[:2] == (3, pytest.approx(2 / 9))      # 0.7 lies before it
    assert B.sample(l, [9, 9, 1, 1e-6], top_p=0.65)[0] == 2
    assert B.sample(l, [9, 1e-9, 1, 1e-6], min_p=0.45)[:2] == (3, pytest.approx(2 / 9))
    assert B.sample(l, [9, 1, 1, 1], temperature=0)[:2] == (0, 1.0)
    assert B.sample([1.0, 1.0, 1.0], [3, 2, 1], top_k=2)[0] == 1                           # the lowest of equals
    for bad in ([math.nan, 1.0], [math.inf, 1.0], [-math.inf, -math.inf]):
        assert B.sample(bad, [1, 1])[:2] == (-1, 0.0)


def test_sample_distribution():
    g = np.random.default_rng(2)
    l = np.log([0.5, 0.25, 0.15, 0.1])
    n = 4000
    got = np.bincount([B.sample(l, g.exponential(size=4), top_k=3)[0] for _ in range(n)], minlength=4) / n
    want = np.array([0.5, 0.25, 0.15, 0.0]) / 0.9
    assert got[3] == 0 and (np.abs(got - want) < 5 * np.sqrt(want * (1 - want) / n) + 1e-9).all()

"""The 64-bit references of the operators around the layers, against differences and known values (CPU)."""
import numpy as np
import pytest

from oracle import model_ops as M


def difference(loss, a, at, h=1e-5):
    up, down = a.copy(), a.copy()
    up[at] += h
    down[at] -= h
    return (loss(up) - loss(down)) / (2 * h)


@pytest.mark.parametrize("K", [1, 2, 4])
@pytest.mark.parametrize("L", [1, 2, 6])
@pytest.mark.parametrize("silu", [True, False])
def test_conv_gradient_is_the_slope(K, L, silu):
    r = np.random.default_rng(K * 10 + L)
    B, D = 2, 3
    a = dict(x=r.standard_normal((B, D, L)), w=r.standard_normal((D, K)), bias=r.standard_normal(D),
             state=r.standard_normal((B, D, K - 1)))
    dy, dso = r.standard_normal((B, D, L)), r.standard_normal((B, D, K - 1))
    g = M.conv_grad(a["x"], a["w"], dy, a["bias"], a["state"], dso, silu)

    def loss(**over):
        y, s = M.conv(**dict(a, **over), silu=silu)
        return (y * dy).sum() + (s * dso).sum()
    for name, gname in (("x", "dx"), ("w", "dw"), ("bias", "dbias"), ("state", "dstate")):
        for at in np.ndindex(*a[name].shape):
            assert abs(difference(lambda v: loss(**{name: v}), a[name], at) - g[gname][at]) < 1e-8


def test_embedding_gradient_is_the_slope():
    r = np.random.default_rng(1)
    tokens, W, dy = np.array([2, 0, 2, -1, 3, 7]), r.standard_normal((4, 3)), r.standard_normal((6, 3))
    g = M.embedding_grad(tokens, dy, 4, 1.5)
    assert np.isnan(M.embedding(tokens, W)[5]).all() and (M.embedding(tokens, W)[3] == 0).all()
    for at in np.ndindex(4, 3):
        d = difference(lambda v: np.nansum(M.embedding(tokens, v, 1.5) * dy), W, at)
        assert abs(d - g[at]) < 1e-8


def test_clip():
    n, (a, b) = M.clip([np.array([3.0]), np.array([[0.0, 4.0]])], 1.0, 0.0)
    assert n == 5.0 and np.allclose(a, 0.6) and np.allclose(b, [[0.0, 0.8]])
    assert M.clip([np.array([3.0, 4.0])], 6.0)[1][0].tolist() == [3.0, 4.0]


@pytest.mark.parametrize("with_q", [True, False])
def test_verify_sample_keeps_the_target_distribution(with_q):
    """The first token out (the drafted one if it passes, else the next one) is distributed as the target's.
    Bound: 5 standard deviations of each of 4 frequencies over 20,000 draws."""
    r = np.random.default_rng(3 + with_q)
    B, V = 20000, 4
    lt, ld = np.array([0.3, 1.2, -0.5, 0.1]), np.array([1.0, 0.0, 0.4, -1.0])
    p, q = M.softmax(lt), M.softmax(ld)
    draft = r.choice(V, size=(B, 1), p=q if with_q else [1.0, 0, 0, 0])
    logits = np.broadcast_to(lt, (B, 2, V))
    acc, nxt, probs, _ = M.verify_sample(logits, draft, r.random((B, 1)), r.exponential(size=(B, V)),
                                         np.broadcast_to(ld, (B, 1, V)) if with_q else None)
    first = np.where(acc == 1, draft[:, 0], nxt)
    freq = np.bincount(first, minlength=V) / B
    assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / B)).all()
    assert np.allclose(probs[:, 0], p[draft[:, 0]])

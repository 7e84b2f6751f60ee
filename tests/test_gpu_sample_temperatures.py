"""The sampling's weights at the largest and smallest temperatures, in rows of every kernel.

Two tokens race, the others are masked.  A weight is within 1e-5 of its own for exponents of a few units, and with T near fp32's largest value the
fp32 inverse is subnormal and adds 2^-150 of 2^-128 (2.4e-7 per unit of the exponent); the tolerance is that of test_gpu_sample.py."""
import math

import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
VOCABS = [60, 256, 600, 3000, 9000, 2 ** 20 + 5]
TOL = 2e-5


def shares(V, logits, temperature, **kw):
    """The probabilities that two tokens are drawn with, by noise that lets the one or the other win."""
    import paper_2401_13660_amd as mb
    l = torch.full((2, V), -math.inf, device="cuda:0")
    l[:, 10:12] = torch.tensor(logits)
    noise = torch.ones(2, V, device="cuda:0")
    noise[0, 10] = noise[1, 11] = 1e-30
    token, prob = mb.sample(l, noise, temperature=temperature, return_prob=True, **kw)
    assert token.tolist() == [10, 11]
    t = torch.full((2,), temperature, device="cuda:0")
    again, prob2 = mb.sample(l, noise, temperature=t, return_prob=True, **kw)
    assert torch.equal(token, again) and torch.equal(prob, prob2)
    return prob.tolist()


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("logits,temperature", [((3e38, -3e38), 3e38), ((3e38, -3e38), 1e38), ((3.4e38, -3.4e38), 3.4e38), ((-1e38, 3.3e38), 2e38),
                                                ((1.0, -1.0), 1.0), ((0.5, -3.0), 1.0001), ((0.5, -3.0), 0.9999)])
def test_largest(V, logits, temperature):
    announce(f"sample of {V} at temperature {temperature}")
    a, b = (float(torch.tensor(v, dtype=torch.float32)) for v in logits)
    t = float(torch.tensor(temperature, dtype=torch.float32))
    want = [1 / (1 + math.exp((b - a) / t)), 1 / (1 + math.exp((a - b) / t))]
    for kw in (dict(), dict(top_p=0.9999999), dict(top_k=5)):
        for got, ref in zip(shares(V, logits, temperature, **kw), want):
            assert abs(got - ref) <= TOL * ref, kw


@pytest.mark.parametrize("V", VOCABS)
def test_smallest(V):
    """Down to 2^-127, subnormal temperatures and logits; below it they are refused, as numbers and row by row."""
    import paper_2401_13660_amd as mb
    for temperature, other in ((2.0 ** -126, -2.0 ** -126), (2.0 ** -127 * 1.01, -2.0 ** -128), (6e-39, -9e-39), (1e-30, -2e-30)):
        announce(f"sample of {V} at temperature {temperature}")
        t, b = (float(torch.tensor(v, dtype=torch.float32)) for v in (temperature, other))
        want = [1 / (1 + math.exp(b / t)), 1 / (1 + math.exp(-b / t))]
        for got, ref in zip(shares(V, (0.0, other), temperature), want):
            assert abs(got - ref) <= TOL * ref
    logits, noise = torch.zeros(2, V, device="cuda:0"), torch.ones(2, V, device="cuda:0")
    for temperature in (2.0 ** -127, 4e-39, 3e-39):
        with pytest.raises(mb.MBScanError):
            mb.sample(logits, noise, temperature=temperature)
        t = torch.tensor([temperature, 1.0], device="cuda:0")
        token, prob = mb.sample(logits, noise, temperature=t, return_prob=True)
        assert token.tolist() == [-1, 0] and prob[0] == 0

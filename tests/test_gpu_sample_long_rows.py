"""GPU parity of the filtered sampling on rows of about 2^20 tokens and more, whose weights can sum to more than 2^20.

Equal logits have weights of exactly 1 and sums of whole numbers, so that which tokens a filter keeps is known: top-p keeps those with
i < p V, the product taken exactly.  Their probability is one quotient in 64 bits, rounded to fp32 (2^-24; twice that is allowed).  Other rows are checked as
in test_gpu_sample.py, whose tolerances hold for rows of any length: weights are fp32, their sum is taken in whole numbers."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_sample import check, inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
LENGTHS = [2 ** 20 - 1, 2 ** 20, 2 ** 20 + 3, 1500001, 2 ** 22]


@pytest.mark.parametrize("V", LENGTHS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits(V, dtype):
    import paper_2401_13660_amd as mb
    announce(f"sample of {V} equal logits {dtype}")
    logits = torch.full((1, V), -1.5, device="cuda:0", dtype=dtype)
    for keep in (1, V // 4 + 1, V // 2, V - 1, V):
        p = float(np.float32((keep - 0.5) / V))
        for kw, n in ((dict(top_k=keep), keep), (dict(top_p=p), math.ceil(Fraction(p) * V)), (dict(), V),
                      (dict(top_k=keep, top_p=0.5), math.ceil(Fraction(keep, 2)))):
            noise = torch.ones(1, V, device="cuda:0")
            noise[:, n - 1] = 1e-3                              # the last one kept wins
            noise[:, n:] = 1e-6                                 # those after it would
            token, prob = mb.sample(logits, noise, return_prob=True, **kw)
            assert int(token) == n - 1, (keep, kw)
            assert abs(float(prob) * n - 1) <= 2.0 ** -23, (keep, kw, float(prob))


@pytest.mark.parametrize("V", [2 ** 20 + 5, 3000001])
def test_settings(V):
    """Flat rows (their weights sum to most of V), ordinary and peaked ones."""
    announce(f"sample of {V} tokens")
    for dtype, temperature in (("f32", 100.0), ("bf16", 3.0), ("f32", 0.3)):
        logits, noise = inputs(2, V, dtype, 7)
        for kw in (dict(), dict(top_p=0.9), dict(top_k=V // 2, top_p=0.7), dict(min_p=0.2, top_p=0.99)):
            check(logits, noise, temperature=temperature, **kw)
    logits[0, :-9] = -math.inf                                  # nine tokens left, and none
    logits[1] = -math.inf
    check(logits, noise, top_p=0.6)
    check(logits, noise, temperature=0.0)


def test_as_shorter_rows():
    """A row made longer by masked tokens, and one among other rows, draw what the short row draws."""
    import paper_2401_13660_amd as mb
    announce("sample of a row and of it among 2^20 masked tokens")
    V = 50000
    short, noise = inputs(3, V, "f32", 5)
    wide = torch.full((3, 2 ** 20 + 1), -math.inf, device="cuda:0")
    far = torch.ones_like(wide)
    wide[:, :V], far[:, :V] = short, noise
    for kw in (dict(top_p=0.8), dict(top_k=70), dict(temperature=2.0)):
        a, p = mb.sample(short, noise, return_prob=True, **kw)
        b, q = mb.sample(wide, far, return_prob=True, **kw)
        # units of 2^-44 of which 50,000 are cut, and finer ones; two roundings to fp32
        assert torch.equal(a, b) and ((p - q).abs() <= 2.0 ** -23 * p).all(), kw


def test_the_longest_rows():
    """2^26 equal logits with a filter, and as many as a row may have."""
    import paper_2401_13660_amd as mb
    V = 2 ** 26
    announce(f"sample of {V} equal logits")
    logits, noise = torch.zeros(1, V, dtype=torch.bfloat16, device="cuda:0"), torch.ones(1, V, device="cuda:0")
    noise[0, V // 2 - 1], noise[0, V // 2:] = 1e-3, 1e-6
    token, prob = mb.sample(logits, noise, top_p=0.5, return_prob=True)
    assert int(token) == V // 2 - 1 and float(prob) * (V // 2) == 1
    V = 2 ** 30 - 1
    announce(f"sample of {V} equal logits")
    logits, noise = torch.zeros(1, V, dtype=torch.bfloat16, device="cuda:0"), torch.ones(1, V, device="cuda:0")
    noise[0, V - 1] = 1e-3
    token, prob = mb.sample(logits, noise, return_prob=True)
    assert int(token) == V - 1 and abs(float(prob) * V - 1) <= 2.0 ** -23

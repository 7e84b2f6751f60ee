"""The sampling's race at the ends of fp32's range: the largest fp32 quotient of weight and noise wins, the lowest index among equal ones.

Two tokens race, the others' noise is infinite.  Quotients are a factor of 2 and more apart."""
import math

import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def race(V, logits, noise, **kw):
    import paper_2401_13660_amd as mb
    l, n = torch.full((1, V), -300.0, device="cuda:0"), torch.full((1, V), math.inf, device="cuda:0")
    l[0, 10:10 + len(logits)], n[0, 10:10 + len(noise)] = torch.tensor(logits), torch.tensor(noise)
    token, prob = mb.sample(l, n, return_prob=True, **kw)
    again = mb.sample(l, n, **kw)
    assert torch.equal(token, again)
    return int(token), float(prob)


VOCABS = [60, 256, 600, 3000, 9000, 2 ** 20 + 5]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("kw", [dict(), dict(top_k=4), dict(top_p=0.999)])
def test_the_ends_of_the_range(V, kw):
    announce(f"sample of {V}: noise near the ends of fp32's range {kw}")
    # subnormal noise: 6.7e36 against 8.3e37; 1.4e38 against 2.5e38; the smallest weight loses to the largest noise
    assert race(V, (-5.0, 0.0), (1e-39, 1.2e-38), **kw)[0] == 11
    assert race(V, (-2.0, 0.0), (1e-39, 4e-39), **kw)[0] == 11
    assert race(V, (0.0, -2.0), (1e-38, 2.0 ** -140), **kw)[0] == 11
    # past fp32's range both are infinite: the lowest index
    assert race(V, (-1.0, 0.0), (1e-39, 2e-39), **kw)[0] == 10
    assert race(V, (-1.0, 0.0), (0.0, 2.0 ** -149), **kw)[0] == 10
    # large noise, quotients of 2^-127 and 2^-126
    assert race(V, (0.0,), (2.0 ** 127,), **kw) == (10, 1.0)
    assert race(V, (0.0, 0.0), (2.0 ** 127, 2.0 ** 126), **kw)[0] == 11
    # a weight of 4e-31 wins where the larger ones' noise is infinite
    token, prob = race(V, (0.0, -70.0), (math.inf, 1.0))
    assert token == 11 and abs(prob / math.exp(-70.0) - 1) <= 2e-5


@pytest.mark.parametrize("V", [60, 3000, 9000])
def test_as_verification(V):
    """verify_sample's token without drafts, for noise of any size."""
    import paper_2401_13660_amd as mb
    announce(f"sample of {V} against verify_sample, noise of any size")
    g = torch.Generator(device="cuda:0").manual_seed(3)
    logits = torch.randn(200, V, generator=g, device="cuda:0") * 3
    # exponents from 2^-149 to 2^120, a factor of their own for each row
    noise = torch.rand(200, V, generator=g, device="cuda:0") + 0.5
    noise = (noise.double() * torch.exp2(torch.randint(-149, 100, (200, 1), generator=g, device="cuda:0").double())
             * torch.exp2(torch.randint(0, 20, (200, V), generator=g, device="cuda:0").double())).float()
    none = torch.zeros(200, 0, device="cuda:0")
    ref = mb.verify_sample(logits[:, None].contiguous(), none.int(), none, noise)[2]
    got = mb.sample(logits, noise)
    # a row is passed over where its two best quotients are within 2e-5, or past fp32's range
    score = torch.exp((logits - logits.amax(1, keepdim=True)).double()) / noise.double()
    best = score.topk(2, dim=1).values
    clear = (best[:, 0] < 3e38) & (best[:, 0] > best[:, 1] * (1 + 2e-5))
    assert clear.sum() >= 100
    assert torch.equal(got[clear], score.argmax(1).int()[clear]) and torch.equal(got[clear], ref[clear])

"""GPU parity of the filtered sampling against 64 bits.

A weight exp((l - max) / T) in fp32 is within (|x| + 4) 2^-23 of its value for an exponent x, below 1e-5 for the weights that
can matter (those above e^-80), and sums of weights are relatively as near.  A sequence whose race is closer than two of them (2e-5), or whose
token changes where top-p or min-p moves by 1e-5 of itself, may come out either way and is passed over; ties are no close
calls, and tests of borders are built of weights that are exact.  prob is the quotient of a weight and a sum (2e-5) and lies
between those that the moved settings give."""
import math

import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import block_ops as B
from test_gpu_embedding import DT, np64, randn, shifted

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
CLOSE, MOVED, TOL = 2e-5, 1e-5, 2e-5


def inputs(b, V, dtype, seed, spread=2.5):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    noise = torch.empty(b, V, device="cuda:0").exponential_(generator=g).clamp_(min=1e-20)
    return (randn((b, V), seed + 1, "f32") * spread).to(DT[dtype]), noise


def check(logits, noise, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, passed_over=0.1):
    import paper_2401_13660_amd as mb
    kw = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    token, prob = mb.sample(logits, noise, return_prob=True, **kw)
    alone = mb.sample(logits, noise, **kw)
    torch.cuda.synchronize()
    b, V = logits.shape
    assert token.dtype == torch.int32 and token.shape == (b,) and prob.dtype == torch.float32 and torch.equal(token, alone)
    # settings as 32 bits hold them
    each = {k: (v.double().tolist() if isinstance(v, torch.Tensor) else [float(np.float32(v))] * b) for k, v in kw.items()}
    over = 0
    for i in range(b):
        l, n = np64(logits[i]), np64(noise[i])
        t, k, p, m = (each[name][i] for name in ("temperature", "top_k", "top_p", "min_p"))
        may = [B.sample(l, n, t, int(k), q, r) for q in {p, p * (1 - MOVED), p * (1 + MOVED)} for r in {m, m * (1 - MOVED)}]
        if min(o[2] for o in may) < CLOSE or len({o[0] for o in may}) > 1:
            over += 1
            continue
        assert int(token[i]) == may[0][0], f"sequence {i}: {int(token[i])} instead of {may[0][0]}"
        low, high = min(o[1] for o in may), max(o[1] for o in may)
        assert low * (1 - TOL) <= float(prob[i]) <= high * (1 + TOL), f"sequence {i}: {float(prob[i])} instead of {low} to {high}"
    assert over <= passed_over * b + 1
    return token


VOCABS = [1, 2, 63, 64, 65, 255, 256, 257, 1000, 1024, 1025, 5000, 32000, 50257, 131072]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_settings(V, dtype):
    announce(f"sample {V} {dtype}")
    logits, noise = inputs(4, V, dtype, V)
    for kw in (dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=5), dict(top_k=V), dict(top_k=V + 7), dict(top_p=0.9),
               dict(top_p=0.5, temperature=1.3), dict(top_p=0.0), dict(min_p=0.05), dict(min_p=1.0), dict(temperature=0.0),
               dict(temperature=0.8, top_k=max(1, V // 3), top_p=0.95, min_p=0.01)):
        check(logits, noise, **kw)


@pytest.mark.parametrize("V", [256, 3000])
@pytest.mark.parametrize("batch", [1, 3, 32, 300])
def test_batches_and_settings_by_row(V, batch):
    announce(f"sample {batch} sequences of {V}, each with its own settings")
    logits, noise = inputs(batch, V, "f32", batch)
    g = torch.Generator(device="cuda:0").manual_seed(5)
    u = torch.rand(4, batch, generator=g, device="cuda:0")
    t = (u[0] + 0.4) * (u[0] > 0.2)
    k = (u[1] * V * 1.2 * (u[1] > 0.3)).int()
    check(logits, noise, t, k, u[2] * 1.2, u[3] * 0.2 * (u[3] > 0.4))
    check(logits, noise, 0.9, k, 0.9, 0.0)
    check(logits, noise, t, 0, u[2], 0.01)


@pytest.mark.parametrize("V", [7, 256, 1000, 4096, 40000])
def test_ties_at_the_borders(V):
    """Equal logits, whose weights are exactly 1: top-k and top-p keep the lowest indices of them."""
    import paper_2401_13660_amd as mb
    announce(f"sample of {V} equal logits")
    for dtype in (torch.float32, torch.bfloat16):
        logits = torch.full((3, V), -1.5, device="cuda:0", dtype=dtype)
        for keep in sorted({1, 2, V // 4 + 1, V // 2, V - 1, V}):
            noise = torch.ones(3, V, device="cuda:0")
            noise[:, keep - 1] = 1e-3                       # the last one kept wins
            noise[:, keep:] = 1e-6                          # those after it would
            noise[2] = 1.0                                  # all the same: the lowest
            for kw in (dict(top_k=keep), dict(top_p=float(np.float32((keep - 0.5) / V))), dict(top_k=keep, top_p=0.9999999)):
                token, prob = mb.sample(logits, noise, return_prob=True, **kw)
                assert token.tolist() == [keep - 1, keep - 1, 0], kw
                assert (prob.double() - 1.0 / keep).abs().max() <= 1e-6 / keep
        # top-p over what top-k leaves
        if V >= 256:
            noise = torch.ones(3, V, device="cuda:0")
            noise[:, 49], noise[:, 50:] = 1e-3, 1e-6
            assert mb.sample(logits, noise, top_k=100, top_p=0.495).tolist() == [49] * 3


@pytest.mark.parametrize("V", [256, 1000, 5000, 70000])
def test_ties_among_others(V):
    """A few larger logits, many equals at the border scattered over the row, smaller ones between them."""
    import paper_2401_13660_amd as mb
    announce(f"sample of {V} logits with equals at the border")
    g = torch.Generator().manual_seed(3)
    kind = torch.randint(0, 3, (V,), generator=g)
    logits = torch.where(kind == 0, 1.0, torch.where(kind == 1, 0.0, -1.0)).to("cuda:0")[None]
    high, equal = (kind == 0).nonzero()[:, 0], (kind == 1).nonzero()[:, 0]
    for more in (1, 2, len(equal) // 2, len(equal)):
        noise = torch.ones(1, V, device="cuda:0")
        noise[0, equal[more - 1]] = 1e-3
        noise[0, equal[more:]] = 1e-6
        noise[0, kind.to("cuda:0") == 2] = 1e-9
        k = len(high) + more
        mass = len(high) * 1.0 + more * math.exp(-1.0)
        total = len(high) + len(equal) * math.exp(-1.0) + int((kind == 2).sum()) * math.exp(-2.0)
        p = (mass - 0.5 * math.exp(-1.0)) / total
        for kw in (dict(top_k=k), dict(top_p=p)):
            token, prob = mb.sample(logits, noise, return_prob=True, **kw)
            assert int(token) == int(equal[more - 1]), (more, kw)
            assert abs(float(prob) - math.exp(-1.0) / mass) <= TOL * math.exp(-1.0) / mass


def test_zeros_of_both_signs():
    """-0 and +0 are equal logits: the lower index ranks first."""
    import paper_2401_13660_amd as mb
    announce("sample: zeros of both signs")
    for V in (64, 2000):
        logits = torch.full((1, V), -3.0, device="cuda:0")
        logits[0, 3], logits[0, 9] = -0.0, 0.0
        noise = torch.ones(1, V, device="cuda:0")
        noise[0, 9] = 1e-6
        assert int(mb.sample(logits, noise, top_k=1)) == 3 and int(mb.sample(logits, noise, temperature=0.0)) == 3
        assert int(mb.sample(logits, noise, top_k=2)) == 9


@pytest.mark.parametrize("V", [40, 256, 900, 3000, 33000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks(V, dtype):
    """Masked tokens by -infinity and by the type's lowest value; rows that mask leaves nothing or one; rows that are no distribution."""
    import paper_2401_13660_amd as mb
    announce(f"sample with masks {V} {dtype}")
    logits, noise = inputs(9, V, dtype, 11)
    low = torch.finfo(DT[dtype]).min
    logits[0, ::2] = -math.inf
    logits[1] = -math.inf
    logits[2] = -math.inf
    logits[2, V - 1] = -5.0
    logits[3, V // 2] = math.nan
    logits[4, 0] = math.inf
    logits[5] = low
    logits[6, 1:] = low
    logits[7, : V - 3] = -math.inf
    for kw in (dict(), dict(top_k=4), dict(top_p=0.8), dict(min_p=0.1), dict(temperature=0.0), dict(top_k=30, top_p=0.7, min_p=0.01),
               dict(top_p=0.9999999), dict(top_k=V - 1)):
        t = check(logits, noise, passed_over=0.3, **kw)
        assert t[1] == -1 and t[3] == -1 and t[4] == -1 and t[2] == V - 1 and t[6] == 0
        assert torch.isfinite(mb.sample(logits, noise, return_prob=True, **kw)[1]).all()


def test_noise():
    """Noise of zero wins, of NaN and infinity never; a row of them gives nothing; temperature 0 does not look at it."""
    import paper_2401_13660_amd as mb
    announce("sample: zeros, infinities and NaN in the noise")
    for V in (100, 3000):
        logits = torch.zeros(5, V, device="cuda:0")
        noise = torch.ones(5, V, device="cuda:0")
        noise[0, 7] = noise[0, 9] = 0.0
        noise[1, 0], noise[1, 1] = math.nan, 0.5
        noise[2] = math.inf
        noise[3] = math.nan
        assert mb.sample(logits, noise).tolist()[:4] == [7, 1, -1, -1]
        assert mb.sample(logits, noise, temperature=0.0).tolist() == [0] * 5
        token, prob = mb.sample(logits, noise, return_prob=True)
        assert (prob[2:4] == 0).all()


def test_settings_out_of_range():
    """Refused as numbers; as tensors their sequences give nothing and the others are as they were."""
    import paper_2401_13660_amd as mb
    announce("sample: settings out of range")
    for V in (100, 3000):
        logits, noise = inputs(4, V, "f32", 2)
        ref = mb.sample(logits, noise)
        one = torch.ones(4, device="cuda:0")
        for name, bad in (("temperature", -1.0), ("temperature", math.nan), ("temperature", math.inf), ("temperature", 1e-44),
                          ("top_p", math.nan), ("min_p", 1.5), ("min_p", math.nan)):
            v = one * (0.0 if name == "min_p" else 1.0)
            v[1] = bad
            token, prob = mb.sample(logits, noise, return_prob=True, **{name: v})
            assert token[1] == -1 and prob[1] == 0
            assert torch.equal(token[[0, 2, 3]], ref[[0, 2, 3]])
            with pytest.raises(mb.MBScanError):
                mb.sample(logits, noise, **{name: bad})


def test_as_verification_without_drafts():
    """Without filters the token is verify_sample's."""
    import paper_2401_13660_amd as mb
    announce("sample against verify_sample")
    for V in (256, 1000, 9000):
        logits, noise = inputs(50, V, "f32", 4)
        none = torch.zeros(50, 0, device="cuda:0")
        ref = mb.verify_sample(logits[:, None].contiguous(), none.int(), none, noise, temperature=0.8)[2]
        assert torch.equal(mb.sample(logits, noise, temperature=0.8), ref)


@pytest.mark.parametrize("shift", [1, 2, 3, 5])
def test_alignment(shift):
    announce(f"sample at addresses {shift} elements on")
    for V in (255, 256, 3001):
        logits, noise = inputs(3, V, "bf16", 6)
        check(shifted(logits, shift), shifted(noise, shift), top_k=40, top_p=0.9)


def test_extreme_spreads():
    """Weights that underflow, logits near the type's limits, temperatures far from 1."""
    announce("sample: extreme spreads")
    for V in (200, 4000):
        for spread in (1e-3, 60.0, 1e4, 1e30):
            logits, noise = inputs(6, V, "f32", 8, spread)
            for kw in (dict(top_p=0.9), dict(top_k=10), dict(temperature=0.05, top_p=0.99), dict(temperature=50.0, min_p=0.3), dict()):
                check(logits, noise, passed_over=0.5, **kw)


def test_distribution():
    """20,000 draws of a nucleus: each token's share is within 5 standard deviations of its probability."""
    import paper_2401_13660_amd as mb
    announce("sample: 20,000 draws")
    n, V = 20000, 300
    row = randn((1, V), 1, "f32") * 2
    logits, noise = row.expand(n, V).contiguous(), inputs(n, V, "f32", 9)[1]
    got = torch.bincount(mb.sample(logits, noise, top_p=0.9), minlength=V).double().cpu().numpy() / n
    e = np.exp(np64(row[0]) - np64(row[0]).max())
    order = np.argsort(-e, kind="stable")
    before = np.cumsum(e[order]) - e[order]
    p = np.zeros(V)
    p[order[before < 0.9 * e.sum()]] = e[order[before < 0.9 * e.sum()]]
    p /= p.sum()
    assert (got[p == 0] == 0).all() and (np.abs(got - p) <= 5 * np.sqrt(p * (1 - p) / n) + 1e-12).all()


def test_past_32_bits():
    import paper_2401_13660_amd as mb
    announce("sample past 2^31 logits")
    b, V = 17000, 131072
    logits = torch.zeros(b, V, dtype=torch.bfloat16, device="cuda:0")
    noise = torch.ones(b, V, device="cuda:0")
    x, e = inputs(20, V, "bf16", 3)
    logits[-20:], noise[-20:] = x, e
    got = mb.sample(logits, noise, top_p=0.9, top_k=500)
    assert torch.equal(got[-20:], mb.sample(x, e, top_p=0.9, top_k=500)) and (got[:-20] == 0).all()

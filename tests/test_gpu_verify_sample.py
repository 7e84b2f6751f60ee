"""GPU parity of mb_verify_sample against 64 bits.

Accepted counts and tokens are compared exactly where no decision on the way is nearer than 1e-5 (relatively) to falling
otherwise: fp32 probabilities here carry up to about 4e-6 (the exponent's argument, up to 40 with 2^-24 on it twice over,
and the sum).  Probabilities: 1e-5 of themselves."""
import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import model_ops as M
from test_gpu_embedding import DT, np64, shifted

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
NEAR = 1e-5


def case(B, n, V, dtype="f32", drafter="logits", ragged=False, seed=0, spread=2.0):
    r = np.random.default_rng(seed)
    lg = r.standard_normal((B, n + 1, V)) * spread
    dl = lg[:, :n] + 0.3 * r.standard_normal((B, n, V))
    a = dict(logits=torch.from_numpy(lg).to(DT[dtype]).to("cuda:0"), draft_logits=torch.from_numpy(dl).to(DT[dtype]).to("cuda:0"),
             uniform=torch.from_numpy(r.random((B, n)).astype(np.float32)).to("cuda:0"),
             noise=torch.from_numpy(r.exponential(size=(B, V)).astype(np.float32) + 1e-20).to("cuda:0"),
             lengths=None, temperature=0.8)
    race = np64(a["draft_logits"]) / 0.8 - np.log(r.exponential(size=(B, n, V)))
    if drafter is None:
        race, a["draft_logits"] = np64(a["logits"])[:, :n], None
    a["draft"] = torch.from_numpy((race.argmax(2) if V else race[..., 0]).astype(np.int32)).to("cuda:0")
    if ragged:
        a["lengths"] = torch.from_numpy(r.integers(-1, n + 2, B).astype(np.int32)).to("cuda:0")
    return a


def call(a, probs=True):
    import paper_2401_13660_amd as mb
    return mb.verify_sample(a["logits"], a["draft"], a["uniform"], a["noise"], a["draft_logits"], lengths=a["lengths"],
                            temperature=a["temperature"], return_probs=probs)


def check(a, most_near=0.02):
    got = call(a)
    less = call(a, probs=False)
    torch.cuda.synchronize()
    n = {k: v if v is None or isinstance(v, float) else np64(v) for k, v in a.items()}
    with np.errstate(all="ignore"):
        acc, nxt, probs, margin = M.verify_sample(n["logits"], n["draft"], n["uniform"], n["noise"], n["draft_logits"],
                                                  n["lengths"], a["temperature"])
    sure = margin > NEAR
    assert (~sure).mean() <= most_near, "the case leaves too much to rounding"
    assert np.array_equal(got[0].cpu().numpy()[sure], acc[sure]), "accepted differ"
    assert np.array_equal(got[2].cpu().numpy()[sure], nxt[sure]), "next tokens differ"
    assert torch.equal(got[1], got[0] - 1)
    assert (np.abs(np64(got[3]) - probs) <= 1e-5 * np.abs(probs) + 1e-37).all()
    for x, y in zip(less, got):
        assert torch.equal(x, y), "the answer depends on whether probabilities are asked for"
    return acc, nxt


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafter", ["logits", None])
@pytest.mark.parametrize("B,n,V", [(1, 0, 256), (1, 1, 256), (32, 16, 256), (3, 40, 256), (4, 17, 1), (5, 3, 2), (6, 5, 63),
                                   (6, 5, 65), (4, 9, 257), (7, 4, 1000), (3, 4, 1025), (3, 2, 5000), (2, 3, 32000),
                                   (2, 2, 70001), (65, 2, 300)])
def test_shapes(dtype, drafter, B, n, V):
    announce(f"verify_sample ({B}, {n}, {V}) {dtype} drafter={drafter}")
    check(case(B, n, V, dtype, drafter, seed=B + n + V))


@pytest.mark.parametrize("V", [256, 3000])
@pytest.mark.parametrize("drafter", ["logits", None])
def test_ragged(V, drafter):
    """Lengths from below zero to past the end: clamped."""
    announce(f"verify_sample ragged V={V}")
    a = case(24, 6, V, "bf16", drafter, ragged=True, seed=3)
    acc, _ = check(a)
    assert (acc <= np.clip(np64(a["lengths"]), 0, 6)).all()
    a["lengths"].fill_(0)                                   # no drafts: the first row's sample
    acc, nxt = check(a)
    assert (acc == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 256, 2500])
@pytest.mark.parametrize("low", [float("-inf"), None])
def test_masks(dtype, V, low):
    """Masked tokens, by -infinity and by the type's lowest value: never drawn, never passed; rows that mask everything
    by the lowest value stay distributions."""
    announce(f"verify_sample masks {dtype} V={V} low={low}")
    a = case(16, 5, V, dtype, seed=4)
    low = torch.finfo(DT[dtype]).min if low is None else low
    mask = torch.rand(16, 6, V, generator=torch.Generator(device="cuda:0").manual_seed(5), device="cuda:0") < 0.7
    mask[:, :, 3] = False
    a["logits"].masked_fill_(mask, low)
    a["draft_logits"].masked_fill_(mask[:, :5] & (torch.arange(V, device="cuda:0") % 3 == 0), low)
    acc, nxt = check(a)
    gone = mask.cpu().numpy()
    assert not any(gone[b, acc[b], nxt[b]] for b in range(16))
    if low != float("-inf"):
        a["logits"].fill_(low)                              # nothing above the lowest value: uniform
        assert set(check(a)[1] >= 0) == {True}


@pytest.mark.parametrize("V", [256, 1500, 5000])
def test_rows_that_are_no_distribution(V):
    announce(f"verify_sample: rows of -infinity, NaN, +infinity, V={V}")
    a = case(12, 3, V, seed=6)
    inf, nan = float("inf"), float("nan")
    a["uniform"].fill_(0.0)                                 # everything that can pass passes
    a["logits"][0, 0] = -inf
    a["logits"][1, 1, V - 1] = nan
    a["logits"][2, 2, 0] = inf
    a["logits"][3, 3] = -inf                                # the row after the drafts
    a["draft_logits"][4, 0] = -inf
    a["draft_logits"][5, 1, V // 2] = nan
    a["draft_logits"][6, 2, 1] = inf
    a["logits"][7, 0, 0] = nan
    a["draft_logits"][7, 0] = -inf
    a["logits"][8, 1] = nan
    a["logits"][9, 2, :V - 1] = -inf                        # one token left
    a["draft"][9, 2] = V - 1
    acc, nxt = check(a)
    assert acc[:10].tolist() == [0, 1, 2, 3, 0, 1, 2, 0, 1, 3]
    assert nxt[:4].tolist() == [-1] * 4 and (nxt[4:7] >= 0).all() and nxt[7:9].tolist() == [-1, -1]


@pytest.mark.parametrize("V", [256, 4000])
@pytest.mark.parametrize("drafter", ["logits", None])
def test_drafts_outside_the_vocabulary(V, drafter):
    announce(f"verify_sample: drafted tokens outside, V={V}")
    a = case(6, 3, V, drafter=drafter, seed=7)
    a["uniform"].fill_(0.0)
    a["draft"][0, 0], a["draft"][1, 1], a["draft"][2, 2], a["draft"][3, 0] = -1, V, 2 ** 31 - 1, -2 ** 31
    acc, nxt = check(a)
    assert acc[:4].tolist() == [0, 1, 2, 0] and (nxt >= 0).all()


@pytest.mark.parametrize("V", [64, 256, 3000])
def test_nothing_left_of_the_target(V):
    """The drafter's distribution is the target's and a token does not pass (uniform 1): the target itself is drawn from."""
    import paper_2401_13660_amd as mb
    announce(f"verify_sample: equal distributions, V={V}")
    a = case(8, 2, V, seed=8)
    a["draft_logits"] = a["logits"][:, :2].contiguous()
    a["uniform"].fill_(1.0)
    acc, _, nxt = call(a, probs=False)
    torch.cuda.synchronize()
    one = mb.verify_sample(a["logits"][:, :1].contiguous(), a["draft"][:, :0].contiguous(), a["uniform"][:, :0].contiguous(),
                           a["noise"], temperature=0.8)
    assert (acc == 0).all() and torch.equal(nxt, one[2])


@pytest.mark.parametrize("V", [7, 256, 300, 5000])
def test_ties_go_to_the_lowest(V):
    announce(f"verify_sample ties V={V}")
    a = case(3, 0, V, seed=9)
    a["logits"].zero_()
    a["noise"].fill_(2.0)
    a["noise"][1, V // 2:] = 1.0
    a["noise"][2, V - 1] = 0.5
    acc, _, nxt = call(a, probs=False)
    assert nxt.tolist() == [0, V // 2, V - 1]


@pytest.mark.parametrize("V", [255, 256, 3001])
def test_alignment(V):
    announce(f"verify_sample at odd addresses V={V}")
    a = case(5, 4, V, "bf16", seed=10)
    got = call(a)
    b = {k: shifted(v, 1) if isinstance(v, torch.Tensor) else v for k, v in a.items()}
    for x, y in zip(got, call(b)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("V", [5, 1030])
@pytest.mark.parametrize("drafter", [True, False])
def test_distribution(V, drafter):
    """What comes first, the drafted token if it passes and else the next one, is distributed as the target's samples:
    5 standard deviations of each of five classes' frequencies over 40,000 sequences."""
    import paper_2401_13660_amd as mb
    announce(f"verify_sample: distribution of the first token, V={V}, drafter={drafter}")
    B = 40000 if V < 100 else 8000
    g = torch.Generator(device="cuda:0").manual_seed(11)
    lt, ld = torch.randn(V, generator=g, device="cuda:0"), torch.randn(V, generator=g, device="cuda:0")
    p, q = lt.double().softmax(0), ld.double().softmax(0)
    draft = torch.multinomial(q if drafter else p, B, replacement=True, generator=g).int()[:, None].contiguous()
    if not drafter:
        draft.fill_(1)
    acc, _, nxt = mb.verify_sample(lt.expand(B, 2, V).contiguous(), draft, torch.rand(B, 1, generator=g, device="cuda:0"),
                                   torch.empty(B, V, device="cuda:0").exponential_(generator=g),
                                   ld.expand(B, 1, V).contiguous() if drafter else None)
    first = torch.where(acc == 1, draft[:, 0], nxt).long() % 5
    freq = torch.bincount(first, minlength=5).double() / B
    p5 = torch.zeros(5, dtype=torch.float64, device="cuda:0").index_add_(0, torch.arange(V, device="cuda:0") % 5, p)
    assert ((freq - p5).abs() < 5 * (p5 * (1 - p5) / B).sqrt()).all()


def test_feeds_the_scan():
    """The state after the last accepted byte, on the device: last_pos goes into the scan as it is."""
    import paper_2401_13660_amd as mb
    from gpu_util import to_device
    from paper_2401_13660_amd.inputs import make_inputs
    announce("verify_sample: last_pos into scan_fwd's positions")
    t = to_device(make_inputs(6, 64, 12, 16, dtype="bf16", seed=12, with_h0=True))
    a = case(6, 12, 256, seed=13)
    acc, last, _ = call(a, probs=False)
    args = (t["u"], t["delta"], t["A"], t["B"], t["C"])
    kw = dict(D=t["Dskip"], dt_bias=t["dt_bias"], z=t["z"], h0=t["h0"])
    _, h_at = mb.scan_fwd(*args, positions=last[None], **kw)
    pos = acc.cpu() - 1
    for b in range(6):
        _, ref = mb.scan_fwd(*args, positions=torch.full((1, 6), int(pos[b]), dtype=torch.int32, device="cuda:0"), **kw)
        assert torch.equal(h_at[0, b], ref[0, b])


def test_refusals():
    import paper_2401_13660_amd as mb
    announce("verify_sample: refusals")
    a = case(2, 3, 16, seed=14)
    for over in (dict(draft=a["draft"].long()), dict(uniform=a["uniform"].double()), dict(noise=a["noise"][:, :8]),
                 dict(draft_logits=a["draft_logits"].bfloat16()), dict(draft_logits=a["logits"]),
                 dict(lengths=a["draft"][:, 0].contiguous()[:1]), dict(temperature=0.0), dict(temperature=float("nan")),
                 dict(logits=a["logits"].half()), dict(logits=a["logits"].transpose(1, 2)), dict(draft=a["draft"].cpu())):
        with pytest.raises(mb.MBScanError):
            call(dict(a, **over))

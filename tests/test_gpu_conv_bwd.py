"""GPU parity of the convolution's gradient against 64 bits.

Tolerances, with inputs of unit variance and weights within 1/2: the pre-activation is a sum of up to 5 terms, so it is
off by at most 5 2^-24 (|bias| + sum |w x|), 3e-6 at |x| <= 5; the slope of the Swish changes by at most half of that and
carries about 1e-6 of the exponential and the reciprocal: 3e-6 of |dy| <= 5.  dx sums up to 4 of those with weights whose
magnitudes sum to 2 at most: 5e-5 beside an rms of about 0.4 (rel_err: a bf16 result adds its rounding, 2^-8).  dw and
dbias sum n = batch L of them: (6e-6 + n 2^-24) of the sum of the magnitudes |dy ext|."""
import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import model_ops as M
from parity import rel_err
from test_gpu_embedding import DT, np64, randn, shifted

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
TOL = 5e-5


def inputs(B, D, L, K, dtype, out, seed, state=True):
    r = {"x": randn((B, D, L), seed, dtype), "dy": randn((B, D, L), seed + 1, out),
         "w": (torch.rand(D, K, generator=torch.Generator().manual_seed(seed)) - 0.5).to("cuda:0"),
         "bias": (torch.rand(D, generator=torch.Generator().manual_seed(seed + 1)) - 0.5).to("cuda:0"),
         "state": None, "dstate_out": None}
    if state:
        r["state"], r["dstate_out"] = randn((B, D, K - 1), seed + 2, "f32"), randn((B, D, K - 1), seed + 3, "f32")
    return r


def call(a, silu=True):
    import paper_2401_13660_amd as mb
    return mb.conv1d_bwd(a["x"], a["w"], a["dy"], a["bias"], a["state"], a["dstate_out"], apply_silu=silu)


def check(a, silu=True):
    g, again = call(a, silu), call(a, silu)
    torch.cuda.synchronize()
    n = {k: None if v is None else np64(v) for k, v in a.items()}
    args = (n["bias"], n["state"], n["dstate_out"], silu)
    ref = M.conv_grad(n["x"], n["w"], n["dy"], *args)
    # magnitudes: |dy| times |ext|, from the gradient of a convolution without bias, state or Swish in them
    mag = M.conv_grad(np.abs(n["x"]), n["w"], np.abs(n["dy"]), None, None if n["state"] is None else np.abs(n["state"]), None,
                      False)
    terms = 6e-6 + a["x"].shape[0] * a["x"].shape[2] * 2.0 ** -24
    for k in g:
        if g[k] is None:
            assert a["bias"] is None
            continue
        assert torch.equal(g[k], again[k]), f"two calls differ in {k}"
        got = np64(g[k])
        assert got.shape == ref[k].shape
        if k in ("dw", "dbias"):
            bad = np.abs(got - ref[k]) > terms * mag[k] * 1.2
            assert not bad.any(), f"{k}: {bad.sum()} off, {np.abs(got - ref[k]).max():.2e}"
        elif got.size:
            tol = TOL + (2.0 ** -8 if k == "dx" and a["dy"].dtype == torch.bfloat16 else 0.0)
            # differences are measured against the tensor's own values or a unit gradient's, whichever is more
            err = np.max(np.abs(got - ref[k]) / (np.abs(ref[k]) + max(0.4, np.sqrt(np.mean(ref[k] ** 2)))))
            assert err <= tol, f"{k}: {err:.2e}"
    return g


@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("L", [1, 2, 3, 5, 8, 64, 259, 520])
def test_lengths(K, dtype, out, L):
    announce(f"conv1d_bwd (2, 5, {L}) K={K} {dtype} {out}")
    check(inputs(2, 5, L, K, dtype, out, 100 * K + L))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,D,L", [(1, 1, 4099), (3, 7, 1021), (1, 300, 513), (2, 2, 9000), (5, 64, 16), (1, 3, 20480)])
def test_shapes(dtype, B, D, L):
    announce(f"conv1d_bwd ({B}, {D}, {L}) {dtype}")
    check(inputs(B, D, L, 4, dtype, dtype, B + D + L))


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("state", [True, False])
def test_options(silu, bias, state):
    announce(f"conv1d_bwd silu={silu} bias={bias} state={state}")
    a = inputs(2, 9, 77, 4, "f32", "f32", 7, state)
    if not bias:
        a["bias"] = None
    check(a, silu)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [512, 1027])
def test_alignment(dtype, L):
    announce(f"conv1d_bwd at odd addresses {dtype} L={L}")
    a = inputs(2, 3, L, 4, dtype, dtype, 8)
    g = check(a)
    b = {k: v if v is None else shifted(v, 1 + i) for i, (k, v) in enumerate(a.items())}
    h = call(b)
    torch.cuda.synchronize()
    for k in g:
        assert torch.equal(g[k], h[k]), k


def test_empty():
    announce("conv1d_bwd without timesteps or rows")
    a = inputs(2, 3, 0, 4, "f32", "f32", 9)
    g = call(a)
    torch.cuda.synchronize()
    assert (g["dw"] == 0).all() and (g["dbias"] == 0).all() and torch.equal(g["dstate"], a["dstate_out"])
    a["dstate_out"] = None
    assert (call(a)["dstate"] == 0).all()
    g = call(inputs(0, 3, 5, 4, "f32", "f32", 9))
    torch.cuda.synchronize()
    assert (g["dw"] == 0).all() and (g["dbias"] == 0).all()


def test_large_arguments():
    """Far from zero the Swish is flat or the identity: slopes 0 and 1, no NaN."""
    announce("conv1d_bwd: pre-activations of +-1e4 and more")
    x = torch.tensor([[[1e4, -1e4, 3e38, -3e38, 88.0, -88.0, 200.0, -200.0]]], device="cuda:0")
    a = dict(x=x, w=torch.ones(1, 1, device="cuda:0"), dy=torch.ones_like(x), bias=None, state=None, dstate_out=None)
    g = call(a)
    torch.cuda.synchronize()
    assert np.allclose(np64(g["dx"])[0, 0], [1, 0, 1, 0, 1, 0, 1, 0], atol=1e-6)


def test_a_nan_stays_near_its_input():
    """A NaN input spoils the outputs that its taps reach and the channel's dw, nothing else."""
    announce("conv1d_bwd: a NaN")
    a = inputs(2, 4, 1100, 4, "bf16", "bf16", 10)
    clean = call(a)
    a["x"] = a["x"].clone()
    a["x"][1, 2, 700] = float("nan")
    g = call(a)
    torch.cuda.synchronize()
    bad = torch.isnan(g["dx"][1, 2]).nonzero().flatten().tolist()
    assert bad == list(range(697, 704))
    for k in ("dx", "dw", "dbias"):
        other = torch.isnan(g[k])
        assert torch.equal(torch.where(other, clean[k], g[k]), clean[k]), k
    assert torch.isnan(g["dw"]).nonzero()[:, 0].unique().tolist() == [2]


def test_autograd_matches_the_layer_and_differences():
    import paper_2401_13660_amd as mb
    announce("causal_conv1d: autograd, and differences in 64 bits")
    a = inputs(2, 3, 40, 4, "f32", "f32", 11)
    t = {k: a[k].clone().requires_grad_() for k in ("x", "w", "bias", "state")}
    y, s = mb.causal_conv1d(t["x"], t["w"], t["bias"], t["state"])
    ((y * a["dy"]).sum() + (s * a["dstate_out"]).sum()).backward()
    n = {k: np64(v) for k, v in a.items()}

    def loss(**over):
        v = {k: n[k] for k in ("x", "w", "bias", "state")}
        v.update(over)
        y, s = M.conv(**v)
        return (y * n["dy"]).sum() + (s * n["dstate_out"]).sum()
    r = np.random.default_rng(12)
    for k in t:
        for _ in range(6):
            at = tuple(int(r.integers(m)) for m in n[k].shape)
            up, down = n[k].copy(), n[k].copy()
            up[at] += 1e-5
            down[at] -= 1e-5
            slope = (loss(**{k: up}) - loss(**{k: down})) / 2e-5
            # dw sums 80 terms of at most 25: 80 * 3e-6 * 25
            assert abs(slope - float(t[k].grad[at])) <= (6e-3 if k in ("w", "bias") else 1e-3), k
    # an unused output has no gradient
    y2, _ = mb.causal_conv1d(t["x"], t["w"], t["bias"], t["state"])
    g = torch.autograd.grad(y2, [t["x"], t["state"]], a["dy"])
    a["dstate_out"] = None
    ref = call(a)
    assert torch.equal(g[0], ref["dx"]) and torch.equal(g[1], ref["dstate"])
    _, s3 = mb.causal_conv1d(t["x"], t["w"], t["bias"], t["state"])
    g = torch.autograd.grad(s3.sum(), t["x"])[0]
    assert (g[:, :, :-3] == 0).all() and (g[:, :, -3:] == 1).all()


def test_layer_size():
    """The 972M layer's rows at a fifth of its context, channels sampled."""
    announce("conv1d_bwd (4, 3584, 1640) bf16")
    a = inputs(4, 3584, 1640, 4, "bf16", "bf16", 13, state=False)
    g = call(a)
    rows = torch.tensor([0, 1, 63, 64, 1791, 3583], device="cuda:0")
    sub = dict(a, x=a["x"][:, rows].contiguous(), dy=a["dy"][:, rows].contiguous(), w=a["w"][rows].contiguous(),
               bias=a["bias"][rows].contiguous())
    ref = M.conv_grad(np64(sub["x"]), np64(sub["w"]), np64(sub["dy"]), np64(sub["bias"]))
    assert rel_err(np64(g["dx"][:, rows]), ref["dx"]) <= TOL + 2.0 ** -8
    assert rel_err(np64(g["dw"][rows]), ref["dw"]) <= 1e-3
    assert rel_err(np64(g["dbias"][rows]), ref["dbias"]) <= 1e-3


def test_refusals():
    import paper_2401_13660_amd as mb
    announce("conv1d_bwd: refusals")
    a = inputs(2, 4, 16, 4, "f32", "f32", 14)
    for over in (dict(dy=a["dy"][:, :, :15]), dict(dy=a["dy"].half()), dict(w=a["w"].bfloat16()), dict(w=a["w"][:3]),
                 dict(bias=a["bias"][:3]), dict(state=a["state"][:, :, :2]), dict(dstate_out=a["dstate_out"].bfloat16()),
                 dict(x=a["x"].transpose(0, 1).contiguous().transpose(0, 1)), dict(w=torch.zeros(4, 5, device="cuda:0"),
                                                                                  state=None, dstate_out=None)):
        with pytest.raises(mb.MBScanError):
            call(dict(a, **over))

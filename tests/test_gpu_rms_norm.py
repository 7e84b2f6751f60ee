"""GPU parity of the norm with the residual's addition, and of its gradients, against 64 bits.

Tolerances, U = 2^-24 being half a step of fp32.  h is one fp32 sum and one rounding: the same bits.  A row's sum of squares
has chains of at most 8 ceil(dim / 512) + 24 positive terms; its root halves that, and mean, root, division and products
add 6 U more.  A 16-bit result adds half of its step.  Gradients: the terms of d as written out below, the row's sum with
its chains; dw sums rows / 256 + 40 terms one after the other at most."""
import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import block_ops as B
from test_gpu_embedding import DT, np64, randn, shifted

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
U = 2.0 ** -24


def half(dtype):
    return 0.0 if dtype in ("f32", torch.float32) else torch.finfo(torch.bfloat16).eps / 2


def chain(dim):
    return 8 * -(-dim // 512) + 24


def r_tol(dim):
    return (0.5 * chain(dim) + 6) * U


def inputs(rows, dim, x, res, seed):
    a = dict(x=randn((rows, dim), seed, x), w=randn((dim,), seed + 1, "f32") * 0.2 + 1.0, res=None)
    if res:
        a["res"] = (randn((rows, dim), seed + 2, "f32") * 3).to(DT[res])
    return a


def check_fwd(a, out, eps=1e-5, weighted=True):
    import paper_2401_13660_amd as mb
    x, res, w = a["x"], a["res"], a["w"] if weighted else None
    before = x.clone()
    got = mb.rms_norm_fwd(x, w, res, eps=eps, out_dtype=DT[out], return_rstd=True)
    torch.cuda.synchronize()
    assert torch.equal(before, x)
    h = x if res is None else (x.float() + res.float()).to(res.dtype)
    if res is not None:
        assert torch.equal(got[1], h) and got[1].dtype == res.dtype
    y, rstd = got[0], got[-1]
    assert y.dtype == DT[out] and y.shape == x.shape and rstd.shape == x.shape[:-1]
    ref, r64 = B.rms_norm(np64(h), None if w is None else np64(w), eps)
    dim = x.shape[-1]
    assert (np.abs(np64(rstd) - r64) <= r_tol(dim) * r64).all()
    assert (np.abs(np64(y) - ref) <= (r_tol(dim) + 3 * U + half(out)) * np.abs(ref)).all()
    return got


@pytest.mark.parametrize("dim", [1, 7, 8, 127, 128, 129, 512, 513, 1000, 1024, 1536, 1792, 2048, 2049, 2304, 6144, 6145, 16384, 16385, 40001])
@pytest.mark.parametrize("x,res,out", [("bf16", "f32", "bf16"), ("f32", None, "f32"), ("bf16", "bf16", "f32"), ("f32", "bf16", "bf16"),
                                       ("f32", "f32", "f32"), ("bf16", None, "bf16")])
def test_forward(dim, x, res, out):
    announce(f"rms_norm_fwd dim {dim} x {x} residual {res} out {out}")
    check_fwd(inputs(5, dim, x, res, dim), out)


@pytest.mark.parametrize("rows", [0, 1, 3, 4, 9, 1021, 5000])
def test_rows(rows):
    announce(f"rms_norm_fwd of {rows} rows")
    check_fwd(inputs(rows, 200, "bf16", "f32", 1), "bf16")
    check_fwd(inputs(rows, 2500, "bf16", "f32", 1), "bf16", weighted=False)


@pytest.mark.parametrize("shift", range(1, 8))
def test_alignment(shift):
    announce(f"rms_norm_fwd at addresses {shift} elements on")
    for dim in (1000, 1003):
        a = inputs(3, dim, "bf16", "f32", 5)
        check_fwd({k: shifted(v, shift) for k, v in a.items()}, "bf16")


def test_in_place_and_given():
    import paper_2401_13660_amd as mb
    announce("rms_norm_fwd: h in the residual's place, outputs given")
    for dim in (300, 20000):
        a = inputs(6, dim, "bf16", "f32", 9)
        y, h = mb.rms_norm_fwd(a["x"], a["w"], a["res"])
        stream, out = a["res"].clone(), torch.empty_like(y)
        v = stream._version
        y2, h2 = mb.rms_norm_fwd(a["x"], a["w"], stream, out=out, residual_out=stream)
        torch.cuda.synchronize()
        assert y2 is out and h2 is stream and stream._version > v
        assert torch.equal(y, y2) and torch.equal(h, h2)
        q, s, h3 = mb.rms_norm_fp8(a["x"], a["w"], stream := a["res"].clone(), residual_out=stream)
        torch.cuda.synchronize()
        assert h3 is stream and torch.equal(h, h3)


def test_shapes():
    import paper_2401_13660_amd as mb
    announce("rms_norm_fwd of other shapes")
    x = randn((2, 3, 5, 40), 1, "bf16")
    y, r = mb.rms_norm_fwd(x, return_rstd=True)
    assert y.shape == x.shape and r.shape == (2, 3, 5)
    assert torch.equal(y, mb.rms_norm_fwd(x.view(-1, 40)).view(x.shape))
    assert mb.rms_norm_fwd(x[0, 0, 0]).shape == (40,)
    q, s = mb.rms_norm_fp8(x)
    assert q.shape == x.shape and s.shape == (2, 3, 5, 1)
    for e in (torch.empty(0, 40, device="cuda:0"), torch.empty(4, 0, device="cuda:0")):
        assert mb.rms_norm_fwd(e).shape == e.shape


def test_extremes():
    import paper_2401_13660_amd as mb
    announce("rms_norm_fwd: zeros, NaN, infinities stay in their rows")
    x = randn((6, 300), 3, "f32")
    clean = mb.rms_norm_fwd(x)
    x[1] = 0
    x[2, 7] = float("nan")
    x[4, 299] = float("inf")
    y, r = mb.rms_norm_fwd(x, return_rstd=True)
    q, s = mb.rms_norm_fp8(x)
    torch.cuda.synchronize()
    for i in (0, 3, 5):
        assert torch.equal(y[i], clean[i])
    assert (y[1] == 0).all() and (q[1].float() == 0).all() and torch.isfinite(s[1]).all()
    assert torch.isnan(y[2]).all() and torch.isnan(q[2].float()).all()
    assert r[4] == 0 and torch.isnan(y[4, 299]) and (y[4, :299] == 0).all()
    zero = mb.rms_norm_fwd(torch.zeros(2, 8, device="cuda:0"), eps=0.0)
    assert torch.isnan(zero).all()


@pytest.mark.parametrize("dim", [1, 100, 128, 130, 1792, 2304, 5000, 17000])
@pytest.mark.parametrize("res", [None, "f32", "bf16"])
def test_eight_bits(dim, res):
    """Codes and scales stand for y: a scale is the block's largest over 448, and a value is off by half a step of 8 bits."""
    import paper_2401_13660_amd as mb
    announce(f"rms_norm_fp8 dim {dim} residual {res}")
    a = inputs(7, dim, "bf16", res, 11)
    got = mb.rms_norm_fp8(a["x"], a["w"], a["res"])
    torch.cuda.synchronize()
    h = a["x"] if res is None else (a["x"].float() + a["res"].float()).to(a["res"].dtype)
    if res:
        assert torch.equal(got[2], h)
    y, _ = B.rms_norm(np64(h), np64(a["w"]))
    tol = r_tol(dim) + 6 * U
    top = B.block_tops(y, False)
    s = np64(got[1])
    assert s.shape == top.shape and (np.abs(s - top / 448) <= tol * top / 448).all()
    each = B.widen(s, 7, dim, False)
    back = np64(got[0].float()) * each
    assert (np.abs(back - y) <= (2.0 ** -4 + tol) * np.abs(y) + 2.0 ** -10 * each * (1 + tol)).all()


def grad_inputs(rows, dim, dy, h, seed, dh=True):
    a = dict(dy=randn((rows, dim), seed, dy), h=(randn((rows, dim), seed + 1, "f32") * 2).to(DT[h]), w=randn((dim,), seed + 2, "f32") * 0.2 + 1)
    a["rstd"] = torch.rsqrt(a["h"].float().square().mean(1) + 1e-5)
    a["dh"] = randn((rows, dim), seed + 3, h) if dh else None
    return a


def check_bwd(a, dx_dtype, weighted=True):
    import paper_2401_13660_amd as mb
    w = a["w"] if weighted else None
    call = lambda: mb.rms_norm_bwd(a["dy"], a["h"], a["rstd"], w, a["dh"], dx_dtype=DT[dx_dtype])  # noqa: E731
    g, again = call(), call()
    torch.cuda.synchronize()
    for k in g:
        assert (g[k] is None and again[k] is None) or torch.equal(g[k], again[k]), "two calls differ"
    rows, dim = a["h"].shape
    dy, h, r = np64(a["dy"]), np64(a["h"]), np64(a["rstd"])[:, None]
    w64 = np.ones(dim) if w is None else np64(w)
    ref, dw = B.rms_norm_grad(dy, h, r[:, 0], w64, None if a["dh"] is None else np64(a["dh"]))
    u, gw = h * r, dy * w64
    along, size = np.abs((gw * u).mean(1, keepdims=True)), np.abs(gw * u).mean(1, keepdims=True)
    tol = r * (3 * np.abs(gw) + 5 * np.abs(u) * along + np.abs(u) * size * (chain(dim) + 6)) + 3 * np.abs(ref)
    if a["dh"] is not None:
        tol = tol + np.abs(np64(a["dh"]))
    assert g["dx"].dtype == DT[dx_dtype]
    assert (np.abs(np64(g["dx"]) - ref) <= U * tol + half(dx_dtype) * (np.abs(ref) + U * tol)).all()
    if a["dh"] is not None:
        assert g["dresidual"].dtype == a["h"].dtype
        assert (np.abs(np64(g["dresidual"]) - ref) <= U * tol + half(a["h"].dtype) * (np.abs(ref) + U * tol)).all()
    else:
        assert "dresidual" not in g
    if weighted:
        assert (np.abs(np64(g["dweight"]) - dw) <= (rows / 256 + 43) * U * np.abs(dy * u).sum(0)).all()
    else:
        assert g["dweight"] is None


@pytest.mark.parametrize("dim", [1, 7, 128, 513, 1000, 1536, 1792, 2049, 2304, 6145, 16385])
@pytest.mark.parametrize("dy,h,dx", [("bf16", "f32", "bf16"), ("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"),
                                     ("bf16", "f32", "f32"), ("f32", "f32", "bf16")])
def test_backward(dim, dy, h, dx):
    announce(f"rms_norm_bwd dim {dim} dy {dy} h {h} dx {dx}")
    check_bwd(grad_inputs(6, dim, dy, h, dim), dx)


@pytest.mark.parametrize("rows", [1, 2, 5, 100, 2042, 4100])
@pytest.mark.parametrize("dim", [96, 2500])
def test_backward_rows(rows, dim):
    announce(f"rms_norm_bwd of {rows} rows of {dim}")
    check_bwd(grad_inputs(rows, dim, "bf16", "f32", 3, dh=rows % 2 == 0), "bf16")
    check_bwd(grad_inputs(rows, dim, "f32", "f32", 4, dh=False), "f32", weighted=False)


def test_backward_wide_many():
    """Rows wider than any register kernel's, more of them than workgroups: the sums kept in memory."""
    announce("rms_norm_bwd of 600 rows of 16,400")
    check_bwd(grad_inputs(600, 16400, "bf16", "bf16", 6), "bf16")


def test_backward_nothing():
    import paper_2401_13660_amd as mb
    announce("rms_norm_bwd without rows")
    e = torch.empty(0, 50, device="cuda:0")
    g = mb.rms_norm_bwd(e, e, torch.empty(0, device="cuda:0"), torch.ones(50, device="cuda:0"))
    assert g["dx"].shape == (0, 50) and (g["dweight"] == 0).all()


@pytest.mark.parametrize("res", [True, False])
@pytest.mark.parametrize("weighted", [True, False])
def test_autograd_by_differences(res, weighted):
    """The differentiable operation against central differences in 64 bits of the definition."""
    import paper_2401_13660_amd as mb
    announce("rms_norm's gradients by differences")
    x, w, r = randn((3, 20), 1, "f32"), randn((20,), 2, "f32"), randn((3, 20), 3, "f32")
    cy, ch = randn((3, 20), 4, "f32"), randn((3, 20), 5, "f32")
    leaves = [x.requires_grad_()] + ([w.requires_grad_()] if weighted else []) + ([r.requires_grad_()] if res else [])
    out = mb.rms_norm(x, w if weighted else None, r if res else None, eps=1e-3)
    loss = (out[0] * cy).sum() + (out[1] * ch).sum() if res else (out * cy).sum()
    loss.backward()

    def value(x, w, r):
        h = x + r if res else x
        y = B.rms_norm(h, w if weighted else None, 1e-3)[0]
        return (y * np64(cy)).sum() + ((h * np64(ch)).sum() if res else 0.0)
    at = [np64(t.detach()) for t in (x, w, r)]
    for k, leaf in enumerate((x, w, r)):
        if not any(leaf is t for t in leaves):
            continue
        g = np64(leaf.grad)
        for i in np.ndindex(*g.shape):
            e = [a.copy() for a in at]
            e[k][i] += 1e-5
            up = value(*e)
            e[k][i] -= 2e-5
            assert abs((up - value(*e)) / 2e-5 - g[i]) < 2e-5 * (1 + abs(g[i]))


def test_autograd_parts():
    """Outputs that the loss does not use, inputs that need no gradient, types that differ, a second derivative."""
    import paper_2401_13660_amd as mb
    announce("rms_norm: parts of its gradients")
    x, r = randn((4, 30), 1, "bf16").requires_grad_(), randn((4, 30), 2, "f32").requires_grad_()
    w = torch.ones(30, device="cuda:0", requires_grad=True)
    y, h = mb.rms_norm(x, w, r)
    h.sum().backward()
    assert (x.grad == 1).all() and (r.grad == 1).all() and x.grad.dtype == torch.bfloat16 and (w.grad == 0).all()
    x.grad = r.grad = w.grad = None
    y, h = mb.rms_norm(x, w, r)
    y.float().square().sum().backward()
    first = r.grad.clone()
    y, h = mb.rms_norm(x.detach(), w.detach(), r)
    r.grad = None
    y.float().square().sum().backward()
    assert torch.equal(first, r.grad)
    g, = torch.autograd.grad(mb.rms_norm(r).square().sum(), r, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice|once_differentiable"):
        g.square().sum().backward()


def test_autograd_leaves_of_one_type():
    """Both summands are leaves of one type, or one and the same: gradients in memory of their own, added up over two passes."""
    import paper_2401_13660_amd as mb
    announce("rms_norm: gradients of two leaves")
    x, r = (randn((5, 24), k, "f32").requires_grad_() for k in (1, 2))
    w, c = randn((24,), 3, "f32"), randn((5, 24), 4, "f32")

    def loss(a, b):
        y, h = mb.rms_norm(a, w, b)
        return (y * c).sum() + h.sum()
    loss(x, r).backward()
    once = x.grad.clone()
    assert torch.equal(once, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()
    loss(x, r).backward()
    assert torch.equal(x.grad, 2 * once) and torch.equal(r.grad, 2 * once)
    s = randn((5, 24), 5, "f32").requires_grad_()
    loss(s, s).backward()
    a, b = s.detach().clone().requires_grad_(), s.detach().clone().requires_grad_()
    loss(a, b).backward()
    assert torch.equal(s.grad, a.grad + b.grad)


def test_past_32_bits():
    """Rows past element 2^31, against the rows on their own."""
    import paper_2401_13660_amd as mb
    announce("rms_norm_fwd and rms_norm_bwd past 2^31 elements")
    rows, dim = (1 << 31) // 2048 + 40, 2048
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda:0")
    x[-40:] = randn((40, dim), 8, "bf16")
    y, rstd = mb.rms_norm_fwd(x, return_rstd=True)
    q, s = mb.rms_norm_fp8(x)
    small, r = mb.rms_norm_fwd(x[-40:].clone(), return_rstd=True)
    sq, ss = mb.rms_norm_fp8(x[-40:].clone())
    assert torch.equal(y[-40:], small) and torch.equal(rstd[-40:], r) and torch.equal(s[-40:], ss)
    assert torch.equal(q[-40:].view(torch.uint8), sq.view(torch.uint8))
    del q, y
    g = mb.rms_norm_bwd(x, x, rstd, torch.ones(dim, device="cuda:0"))
    e = mb.rms_norm_bwd(x[-40:].clone(), x[-40:].clone(), r, torch.ones(dim, device="cuda:0"))
    assert torch.equal(g["dx"][-40:], e["dx"])

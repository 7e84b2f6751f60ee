"""Refusals of the norm, the 8-bit matrices and their products, and the sampling, on the CPU: bad arguments are found before
any launch."""
import ctypes
import os

import pytest
import torch

import paper_2401_13660_amd as mb
from paper_2401_13660_amd import _binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmbscan.so not built")

# Fake device addresses: every call with them is invalid and refused, and they are only used without a GPU.
no_gpu_only = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake addresses only on a machine without a GPU")
P = {k: 0x100000000 * (i + 1) for i, k in enumerate(
    ["x", "w", "res", "y", "scales", "h", "rstd", "dy", "dh", "dx", "dres", "dw", "ws", "q", "a", "as", "b", "bs", "c", "logits",
     "noise", "token", "prob", "t", "k", "p", "m"])}
INF, NAN = float("inf"), float("nan")


@no_gpu_only
@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), -2), (dict(dim=-1), -2), (dict(dim=1 << 25), -2), (dict(rows=1 << 50, dim=1 << 20), -2),
    (dict(xt=2), -3), (dict(rt=2), -3), (dict(ot=3), -3), (dict(ot=-1), -3),
    (dict(eps=-1.0), -5), (dict(eps=NAN), -5), (dict(eps=INF), -5),
    (dict(x=None), -1), (dict(y=None), -1), (dict(res=None), -1), (dict(h=None), -1), (dict(ot=2, scales=None), -1),
    (dict(x=P["x"] + 1), -4), (dict(y=P["y"] + 2), -4), (dict(w=P["w"] + 2), -4), (dict(res=P["res"] + 1), -4),
    (dict(h=P["h"] + 2), -4), (dict(rstd=P["rstd"] + 2), -4), (dict(ot=2, scales=P["scales"] + 1), -4),
    (dict(y=P["x"]), -7), (dict(y=P["res"]), -7), (dict(y=P["w"] + 4), -7), (dict(h=P["x"] + 64), -7), (dict(h=P["res"] + 64), -7),
    (dict(rstd=P["y"] + 4), -7), (dict(ot=2, scales=P["x"] + 4), -7), (dict(h=P["y"]), -7),
])
def test_norm_rejects(over, code):
    v = dict(rows=10, dim=64, xt=1, rt=0, ot=0, eps=1e-5, x=P["x"], w=P["w"], res=P["res"], y=P["y"], scales=P["scales"], h=P["h"],
             rstd=P["rstd"])
    v.update(over)
    assert mb.load_library().mb_rms_norm_fwd(*(v[k] for k in ("rows", "dim", "xt", "rt", "ot", "eps", "x", "w", "res", "y", "scales",
                                                              "h", "rstd")), None) == code


def test_norm_empty():
    lib = mb.load_library()
    none = [None] * 8
    assert lib.mb_rms_norm_fwd(0, 64, 0, 0, 0, 1e-5, *none) == 0 and lib.mb_rms_norm_fwd(5, 0, 0, 0, 2, 1e-5, *none) == 0
    assert lib.mb_rms_norm_bwd(0, 64, 0, 0, 0, *[None] * 10) == 0 and lib.mb_rms_norm_bwd(7, 0, 0, 0, 0, *[None] * 10) == 0


@no_gpu_only
@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), -2), (dict(dim=1 << 25), -2), (dict(yt=2), -3), (dict(ht=2), -3), (dict(xt=-1), -3),
    (dict(dy=None), -1), (dict(h=None), -1), (dict(rstd=None), -1), (dict(dx=None), -1),
    (dict(dy=P["dy"] + 2), -4), (dict(h=P["h"] + 1), -4), (dict(dh=P["dh"] + 2), -4), (dict(dx=P["dx"] + 1), -4),
    (dict(dres=P["dres"] + 2), -4), (dict(rstd=P["rstd"] + 2), -4), (dict(w=P["w"] + 1), -4), (dict(dw=P["dw"] + 2), -4),
    (dict(ws=P["ws"] + 8), -4),
    (dict(dx=P["dy"]), -7), (dict(dx=P["h"] + 4), -7), (dict(dres=P["dh"]), -7), (dict(dres=P["dx"]), -7), (dict(dw=P["w"]), -7),
    (dict(dw=P["dx"] + 16), -7), (dict(ws=P["dy"] + 16), -7), (dict(ws=P["dw"]), -7),
])
def test_norm_bwd_rejects(over, code):
    v = dict(rows=10, dim=64, yt=0, ht=0, xt=0, dy=P["dy"], h=P["h"], rstd=P["rstd"], w=P["w"], dh=P["dh"], dx=P["dx"], dres=P["dres"],
             dw=P["dw"], ws=P["ws"])
    v.update(over)
    assert mb.load_library().mb_rms_norm_bwd(*v.values(), None) == code


def test_norm_workspace():
    lib = mb.load_library()
    assert lib.mb_rms_norm_bwd_workspace(-1, 5) == -2 and lib.mb_rms_norm_bwd_workspace(5, 1 << 25) == -2
    assert lib.mb_rms_norm_bwd_workspace(1, 64) == 0 < lib.mb_rms_norm_bwd_workspace(1000, 64)
    assert lib.mb_rms_norm_bwd_workspace(1 << 30, 1792) <= 64 << 20


@no_gpu_only
@pytest.mark.parametrize("over,code", [
    (dict(b=-1), -2), (dict(r=-1), -2), (dict(c=-1), -2), (dict(r=1 << 40), -2), (dict(b=1 << 30, r=1 << 20, c=1 << 20), -2),
    (dict(r=1 << 20, c=1 << 20), -2), (dict(t=2), -3), (dict(x=None), -1), (dict(q=None), -1), (dict(s=None), -1),
    (dict(x=P["x"] + 2), -4), (dict(s=P["scales"] + 1), -4), (dict(q=P["x"]), -7), (dict(q=P["x"] + 399), -7), (dict(s=P["x"] + 4), -7), (dict(s=P["q"]), -7),
])
def test_quantize_rejects(over, code):
    v = dict(b=1, r=10, c=10, t=0, tile=0, tr=0, x=P["x"], q=P["q"], s=P["scales"])
    v.update(over)
    assert mb.load_library().mb_quantize_fp8(*v.values(), None) == code


def test_quantize_empty():
    assert mb.load_library().mb_quantize_fp8(1, 0, 5, 0, 0, 0, None, None, None, None) == 0


@no_gpu_only
@pytest.mark.parametrize("desc,over,code", [
    (None, {}, -1), (dict(batch=-1), {}, -2), (dict(m=-1), {}, -2), (dict(n=1 << 30), {}, -2), (dict(k=1 << 30), {}, -2),
    (dict(m=1 << 29, n=1 << 29), {}, -2), (dict(batch=1 << 40, m=1 << 10, n=1 << 10), {}, -2), (dict(out_dtype=2), {}, -3),
    (dict(reserved=1), {}, -5),
    ({}, dict(a=None), -1), ({}, {"as": None}, -1), ({}, dict(b=None), -1), ({}, dict(bs=None), -1), ({}, dict(c=None), -1),
    ({}, {"as": P["as"] + 2}, -4), ({}, dict(bs=P["bs"] + 1), -4), ({}, dict(c=P["c"] + 2), -4),
    ({}, dict(c=P["a"]), -7), ({}, dict(c=P["b"] + 8), -7), ({}, dict(c=P["as"]), -7), ({}, dict(c=P["bs"]), -7),
])
def test_matmul_rejects(desc, over, code):
    v = {k: P[k] for k in ("a", "as", "b", "bs", "c")}
    v.update(over)
    d = None
    if desc is not None:
        f = dict(batch=2, m=8, n=16, k=64, a_batched=1, b_batched=0, a_tile=0, b_tile=1, out_dtype=0, reserved=0)
        f.update(desc)
        d = ctypes.byref(B.MatmulDesc(**f))
    assert mb.load_library().mb_matmul_fp8(d, *v.values(), None) == code


def test_matmul_empty():
    d = B.MatmulDesc(1, 0, 16, 64, 0, 0, 0, 0, 0, 0)
    assert mb.load_library().mb_matmul_fp8(ctypes.byref(d), *[None] * 6) == 0


@no_gpu_only
@pytest.mark.parametrize("over,code", [
    (dict(b=-1), -2), (dict(V=0), -2), (dict(V=1 << 30), -2), (dict(b=1 << 22), -2), (dict(dt=2), -3),
    (dict(T=-1.0), -5), (dict(T=NAN), -5), (dict(T=INF), -5), (dict(T=1e-44), -5), (dict(tp=NAN), -5), (dict(mp=NAN), -5), (dict(mp=1.5), -5),
    (dict(logits=None), -1), (dict(noise=None), -1), (dict(token=None), -1),
    (dict(logits=P["logits"] + 2), -4), (dict(noise=P["noise"] + 1), -4), (dict(token=P["token"] + 2), -4), (dict(prob=P["prob"] + 2), -4),
    (dict(t=P["t"] + 2), -4), (dict(k=P["k"] + 2), -4), (dict(p=P["p"] + 1), -4), (dict(m=P["m"] + 2), -4),
    (dict(token=P["logits"] + 4), -7), (dict(token=P["noise"]), -7), (dict(prob=P["token"]), -7), (dict(prob=P["t"]), -7), (dict(token=P["k"]), -7),
])
def test_sample_rejects(over, code):
    v = dict(b=4, V=100, dt=0, T=1.0, tk=0, tp=1.0, mp=0.0, t=P["t"], k=P["k"], p=P["p"], m=P["m"], logits=P["logits"], noise=P["noise"],
             token=P["token"], prob=P["prob"])
    if set(over) & {"T", "tp", "mp"}:
        v.update(t=None, p=None, m=None)
    v.update(over)
    assert mb.load_library().mb_sample(*v.values(), None) == code


def test_sample_empty():
    assert mb.load_library().mb_sample(0, 5, 0, 1.0, 0, 1.0, 0.0, *[None] * 9) == 0


def test_binding_refuses():
    """Tensors of the wrong kind, shape, type or place raise; on the CPU all of them are in the wrong place."""
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for call in (lambda: mb.rms_norm_fwd(None), lambda: mb.rms_norm_fwd(x), lambda: mb.rms_norm_fp8(x, w), lambda: mb.rms_norm_fwd(torch.zeros(())),
                 lambda: mb.rms_norm_bwd(x, x, w), lambda: mb.rms_norm_bwd(None, None, None), lambda: mb.quantize_fp8(w), lambda: mb.quantize_fp8(x),
                 lambda: mb.matmul_fp8(x, w, x, w), lambda: mb.matmul_fp8(None, w, x, w), lambda: mb.sample(w, w), lambda: mb.sample(x, x),
                 lambda: mb.rms_norm(x), lambda: mb.linear_fp8(x, x)):
        with pytest.raises(mb.MBScanError):
            call()

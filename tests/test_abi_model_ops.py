"""Refusals of the entry points around the layers, on the CPU: bad arguments are found before any launch."""
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
    ["tokens", "weight", "out", "x", "w", "bias", "state", "dy", "dso", "dx", "dw", "dbias", "dsi", "logits", "dlogits",
     "draft", "lengths", "uniform", "noise", "accepted", "last", "next", "probs", "norm"])}


@no_gpu_only
@pytest.mark.parametrize("name", ["mb_embedding_fwd", "mb_embedding_bwd"])
@pytest.mark.parametrize("over,code", [
    (dict(n=-1), -2), (dict(V=-1), -2), (dict(V=1 << 31), -2), (dict(n=1 << 50, d=1 << 20), -2),
    (dict(tok=3), -3), (dict(it=2), -3), (dict(ot=-1), -3),
    (dict(a=None), -1), (dict(b=None), -1), (dict(c=None), -1),
    (dict(a=P["tokens"] + 2), -4), (dict(b=P["weight"] + 1), -4), (dict(c=P["out"] + 2), -4),
    (dict(c=P["tokens"]), -7), (dict(c=P["weight"] + 4), -7),
])
def test_embedding_rejects(name, over, code):
    v = dict(n=10, V=256, d=64, tok=1, it=1, ot=0, a=P["tokens"], b=P["weight"], c=P["out"])
    v.update(over)
    fn = getattr(mb.load_library(), name)
    ws = [None] if name.endswith("bwd") else []
    assert fn(v["n"], v["V"], v["d"], v["tok"], v["it"], v["ot"], 1.0, v["a"], v["b"], v["c"], *ws, None) == code


def test_embedding_empty():
    lib = mb.load_library()
    assert lib.mb_embedding_fwd(0, 256, 64, 0, 0, 0, 1.0, None, None, None, None) == 0
    assert lib.mb_embedding_fwd(5, 256, 0, 0, 0, 0, 1.0, None, None, None, None) == 0
    assert lib.mb_embedding_bwd(5, 0, 64, 0, 0, 0, 1.0, None, None, None, None, None) == 0


@no_gpu_only
@pytest.mark.parametrize("desc,over,code", [
    (None, {}, -1),
    (dict(batch=-1), {}, -2), (dict(seqlen=-1), {}, -2), (dict(seqlen=1 << 31), {}, -2), (dict(dim=1 << 31), {}, -2), (dict(dim=1 << 25), {}, -2),
    (dict(in_dtype=5), {}, -3), (dict(out_dtype=5), {}, -3),
    (dict(width=0), {}, -5), (dict(width=5), {}, -5), (dict(reserved=1), {}, -5), (dict(reserved2=1), {}, -5),
    ({}, dict(x=None), -1), ({}, dict(w=None), -1), ({}, dict(dy=None), -1), ({}, dict(dx=None), -1),
    ({}, dict(dw=None), -1), ({}, dict(dbias=None), -1),
    ({}, dict(x=P["x"] + 1), -4), ({}, dict(dy=P["dy"] + 2), -4), ({}, dict(state=P["state"] + 2), -4),
    ({}, dict(dx=P["dy"]), -7), ({}, dict(dx=P["x"] + 16), -7), ({}, dict(dw=P["w"]), -7), ({}, dict(dsi=P["dso"]), -7),
    ({}, dict(dsi=P["dx"] + 64), -7), ({}, dict(ws=P["x"] + 8), -4), ({}, dict(ws=P["dy"] + 16), -7),
])
def test_conv_bwd_rejects(desc, over, code):
    v = {k: P[k] for k in ("x", "w", "bias", "state", "dy", "dso", "dx", "dw", "dbias", "dsi")}
    v.update(dict(ws=None), **over)
    d = None
    if desc is not None:
        c = dict(batch=2, dim=8, seqlen=16, width=4, in_dtype=1, out_dtype=0, apply_silu=1, reserved=0, reserved2=0)
        c.update(desc)
        d = ctypes.byref(B.ConvDesc(**c))
    assert mb.load_library().mb_conv1d_bwd(d, v["x"], v["w"], v["bias"], v["state"], v["dy"], v["dso"], v["dx"], v["dw"],
                                           v["dbias"], v["dsi"], v["ws"], None) == code


def _lists(ptrs, sizes, types):
    n = len(ptrs)
    return (ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*sizes), (ctypes.c_int32 * n)(*types)


A0 = 0x7000000000


@no_gpu_only
@pytest.mark.parametrize("count,ptrs,sizes,types,norm,code", [
    (-1, [A0], [4], [0], P["norm"], -2),
    (1, [A0], [-4], [0], P["norm"], -2),
    (2, [A0, 2 * A0], [1 << 55, 1 << 56], [0, 0], P["norm"], -2),
    (1, [A0], [4], [2], P["norm"], -3),
    (1, [None], [4], [0], P["norm"], -1),
    (1, [A0], [4], [0], None, -1),
    (1, [A0 + 2], [4], [0], P["norm"], -4),
    (1, [A0 + 1], [4], [1], P["norm"], -4),
    (1, [A0], [4], [0], P["norm"] + 2, -4),
    (1, [A0], [4], [0], A0 + 8, -7),
])
def test_grad_norm_rejects(count, ptrs, sizes, types, norm, code):
    lib = mb.load_library()
    p, s, t = _lists(ptrs, sizes, types)
    assert lib.mb_grad_norm(count, p, s, t, norm, None, None) == code
    assert lib.mb_clip_grad_norm(count, p, None, s, t, 1.0, 1e-6, norm, None, None) == code


@no_gpu_only
@pytest.mark.parametrize("ptrs,out,max_norm,eps,code", [
    ([A0, A0 + 64], None, -1.0, 1e-6, -5),
    ([A0, A0 + 64], None, float("nan"), 1e-6, -5),
    ([A0, A0 + 64], None, float("inf"), 1e-6, -5),
    ([A0, A0 + 64], None, 1.0, -1.0, -5),
    ([A0, A0 + 64], None, 1.0, float("nan"), -5),
    ([A0, A0 + 60], None, 1.0, 1e-6, -7),               # 16 floats each: the second starts in the first
    ([A0 + 60, A0], None, 1.0, 1e-6, -7),               # in any order
    ([A0, A0], None, 1.0, 1e-6, -7),                    # the same tensor twice
    ([A0, A0 + 64], [2 * A0, 2 * A0 + 32], 1.0, 1e-6, -7),
    ([A0, A0 + 64], [2 * A0, A0 + 64], 1.0, 1e-6, -7),  # one of them in place
    ([A0, A0 + 640], [A0 + 32, 2 * A0], 1.0, 1e-6, -7),
    ([A0, A0 + 64], [2 * A0, None], 1.0, 1e-6, -1),
    ([A0, A0 + 64], [2 * A0, 3 * A0 + 2], 1.0, 1e-6, -4),
    ([A0, A0 + 64], [2 * A0, P["norm"] - 32], 1.0, 1e-6, -7),
])
def test_clip_rejects(ptrs, out, max_norm, eps, code):
    p, s, t = _lists(ptrs, [16, 16], [0, 0])
    o = None if out is None else (ctypes.c_void_p * 2)(*out)
    assert mb.load_library().mb_clip_grad_norm(2, p, o, s, t, max_norm, eps, P["norm"], None, None) == code


@no_gpu_only
def test_workspaces():
    """Their sizes, and that one which overlaps or is not aligned is refused."""
    lib = mb.load_library()
    assert lib.mb_grad_norm_workspace(-1) == -2 and lib.mb_embedding_bwd_workspace(-1, 1, 1) == -2
    assert lib.mb_embedding_bwd_workspace(1 << 31, 256, 64) == -2
    assert lib.mb_embedding_bwd(1 << 31, 5, 8, 1, 0, 0, 1.0, P["tokens"], P["dy"], P["out"], None, None) == -2
    assert lib.mb_conv1d_bwd_workspace(None) == -1
    d = B.ConvDesc(4, 3584, 8192, 4, 1, 1, 1, 0, 0)
    assert lib.mb_conv1d_bwd_workspace(ctypes.byref(d)) >= 4 * 3584 * 5 * 4
    d.width = 5
    assert lib.mb_conv1d_bwd_workspace(ctypes.byref(d)) == -5
    assert lib.mb_verify_sample_workspace(2, 3, 1024) == 0 < lib.mb_verify_sample_workspace(2, 3, 1025)
    assert lib.mb_verify_sample_workspace(2, 3, 0) == -2 and lib.mb_verify_sample_workspace(1 << 31, 3, 5) == -2
    assert 0 < lib.mb_grad_norm_workspace(1) < lib.mb_grad_norm_workspace(1000)
    e = lambda ws: lib.mb_embedding_bwd(9, 5, 8, 1, 0, 0, 1.0, P["tokens"], P["dy"], P["out"], ws, None)  # noqa: E731
    assert e(P["x"] + 8) == -4 and e(P["out"] + 16) == -7 and e(P["tokens"]) == -7
    p, s, t = _lists([A0], [16], [0])
    for ws, code in ((P["x"] + 8, -4), (A0 + 16, -7), (P["norm"], -7)):
        assert lib.mb_grad_norm(1, p, s, t, P["norm"], ws, None) == code
        assert lib.mb_clip_grad_norm(1, p, None, s, t, 1.0, 0.0, P["norm"], ws, None) == code
    o = (ctypes.c_void_p * 1)(2 * A0)
    assert lib.mb_clip_grad_norm(1, p, o, s, t, 1.0, 0.0, P["norm"], 2 * A0 + 16, None) == -7


@no_gpu_only
@pytest.mark.parametrize("over,code", [
    (dict(b=-1), -2), (dict(n=-1), -2), (dict(V=0), -2), (dict(V=(1 << 31) - 1), -2), (dict(n=(1 << 31) - 1), -2),
    (dict(b=1 << 31), -2), (dict(b=1 << 22), -2), (dict(b=1 << 20, n=4, V=2000), -2), (dict(b=1 << 30, n=1 << 20, V=1 << 20), -2), (dict(dt=2), -3),
    (dict(T=0.0), -5), (dict(T=-1.0), -5), (dict(T=float("nan")), -5), (dict(T=float("inf")), -5), (dict(T=1e-44), -5),
    (dict(logits=None), -1), (dict(noise=None), -1), (dict(draft=None), -1), (dict(uniform=None), -1),
    (dict(accepted=None), -1), (dict(next=None), -1),
    (dict(logits=P["logits"] + 1), -4), (dict(dlogits=P["dlogits"] + 1), -4), (dict(lengths=P["lengths"] + 2), -4),
    (dict(probs=P["probs"] + 1), -4),
    (dict(accepted=P["draft"]), -7), (dict(next=P["accepted"]), -7), (dict(probs=P["uniform"] + 4), -7),
    (dict(last=P["noise"]), -7), (dict(next=P["logits"] + 64), -7),
    (dict(ws=P["x"] + 8, V=2000), -4), (dict(ws=P["noise"], V=2000), -7), (dict(ws=P["next"], V=2000), -7),
])
def test_verify_sample_rejects(over, code):
    v = dict(P, b=2, n=3, V=256, dt=1, T=1.0)
    v.update(over)
    assert mb.load_library().mb_verify_sample(
        v["b"], v["n"], v["V"], v["dt"], v["T"], v["logits"], v["dlogits"], v["draft"], v["lengths"], v["uniform"],
        v["noise"], v["accepted"], v["last"], v["next"], v["probs"], v.get("ws"), None) == code


def test_binding_refuses_cpu_tensors_and_wrong_arguments():
    t = torch.zeros(4, dtype=torch.int32)
    f = torch.zeros(2, 3)
    for call in (lambda: mb.embedding_fwd(t, f), lambda: mb.embedding_bwd(t, torch.zeros(4, 3), 5),
                 lambda: mb.embedding_fwd(t, torch.zeros(3)), lambda: mb.embedding_bwd(t, 1, 5),
                 lambda: mb.embedding_fwd(f, f), lambda: mb.conv1d_bwd(torch.zeros(1, 2, 3), f, torch.zeros(1, 2, 3)),
                 lambda: mb.conv1d_bwd(f, f, f), lambda: mb.grad_norm([]), lambda: mb.grad_norm([f]),
                 lambda: mb.clip_grad_norm([f, 3], 1.0), lambda: mb.clip_grad_norm([], 1.0),
                 lambda: mb.verify_sample(f, t, f, f),
                 lambda: mb.verify_sample(torch.zeros(1, 1, 4), torch.zeros(1, 0, dtype=torch.int32), torch.zeros(1, 0),
                                          torch.zeros(1, 4))):
        with pytest.raises(B.MBScanError):
            call()

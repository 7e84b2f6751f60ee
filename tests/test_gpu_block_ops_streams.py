"""The norm, the 8-bit products and the sampling on other streams than the default one, in HIP graphs, through the native entry
points and through Python, on many rows at once, and as they follow each other in a model's step."""
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import block_ops as B
from test_gpu_embedding import np64, randn
from test_gpu_fastcall import both, watched  # noqa: F401  (fixtures)
from test_gpu_fastcall_model_ops import same
from test_gpu_rms_norm import grad_inputs, inputs
from test_gpu_sample import inputs as logits_of

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def calls(seed):
    """name: (a call that returns tensors)"""
    import paper_2401_13660_amd as mb
    a, wide = inputs(300, 500, "bf16", "f32", seed), inputs(40, 5000, "f32", "bf16", seed)
    g = grad_inputs(2500, 300, "bf16", "f32", seed)
    x = randn((3, 300, 700), seed, "bf16")
    q, s = mb.quantize_fp8(x.view(900, 700))
    few, fs = q[:20].contiguous(), s[:20].contiguous()
    big, bs = mb.quantize_fp8(randn((4200, 512), seed + 1, "bf16"))
    bw, ws = mb.quantize_fp8(randn((4100, 512), seed + 2, "f32"), tile=True)
    w, wss = mb.quantize_fp8(randn((1300, 700), seed + 2, "f32"), tile=True)
    small, large = logits_of(20, 256, "f32", seed), logits_of(20, 30000, "bf16", seed)
    return {
        "norm": lambda: list(mb.rms_norm_fwd(a["x"], a["w"], a["res"], return_rstd=True)),
        "norm_wide": lambda: list(mb.rms_norm_fwd(wide["x"], wide["w"], wide["res"])),
        "norm_fp8": lambda: list(mb.rms_norm_fp8(a["x"], a["w"], a["res"])),
        "norm_bwd": lambda: [t for t in mb.rms_norm_bwd(g["dy"], g["h"], g["rstd"], g["w"], g["dh"]).values()],
        "quantize": lambda: list(mb.quantize_fp8(x)),
        "quantize_turned": lambda: list(mb.quantize_fp8(x, transpose=True)),
        "quantize_tiles": lambda: list(mb.quantize_fp8(x, tile=True, transpose=True)),
        "matmul_few": lambda: [mb.matmul_fp8(few, fs, w, wss)],
        "matmul": lambda: [mb.matmul_fp8(q, s, w, wss, out_dtype=torch.float32)],
        "matmul_large": lambda: [mb.matmul_fp8(bw, ws, big, bs)],
        "sample": lambda: list(mb.sample(*small, top_k=40, top_p=0.9, return_prob=True)),
        "sample_wide": lambda: list(mb.sample(*large, top_p=0.9, min_p=0.001, return_prob=True)),
    }


NAMES = ["norm", "norm_wide", "norm_fp8", "norm_bwd", "quantize", "quantize_turned", "quantize_tiles", "matmul_few", "matmul", "matmul_large",
         "sample", "sample_wide"]


def bits(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t


def test_two_streams():
    announce("block operators on two streams at once")
    sets = [calls(1), calls(2)]
    serial = [{k: [t.clone() for t in s[k]()] for k in NAMES} for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for s, c in zip(streams, sets):
        with torch.cuda.stream(s):
            got.append({k: c[k]() for k in NAMES})
    torch.cuda.synchronize()
    for a, b in zip(got, serial):
        for k in NAMES:
            for x, y in zip(a[k], b[k]):
                assert torch.equal(bits(x), bits(y)), k


@pytest.mark.parametrize("name", NAMES)
def test_graph(name):
    announce(f"HIP graph of {name}")
    call = calls(3)[name]
    ref = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph, held = torch.cuda.CUDAGraph(), {}
    with torch.cuda.graph(graph):
        held["out"] = call()
    for r in range(4):
        call()                                              # eager work between replays
        for t in held["out"]:
            bits(t).fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(held["out"], ref):
            assert torch.equal(bits(x), bits(y)), f"replay {r}"


@pytest.mark.parametrize("name", NAMES)
def test_native_and_python(both, name):  # noqa: F811
    """The native entry points take well-formed calls and give Python's results."""
    announce(f"native {name}")
    call = calls(4)[name]
    with torch.no_grad():
        a, b = both(lambda: tuple(bits(t).clone() for t in call()))
    same(a, b)


def test_native_options(both):  # noqa: F811
    import paper_2401_13660_amd as mb
    announce("native entry points: options")
    a = inputs(7, 130, "bf16", "f32", 1)
    x, w, r = a["x"], a["w"], a["res"]
    out, h = torch.empty_like(x), torch.empty_like(r)
    same(*both(lambda: (mb.rms_norm_fwd(x),)))
    same(*both(lambda: mb.rms_norm_fwd(x, w, out_dtype=torch.float32, return_rstd=True)))
    same(*both(lambda: tuple(t.clone() for t in mb.rms_norm_fwd(x, torch.nn.Parameter(w), r, eps=1, out=out, residual_out=h))))
    same(*both(lambda: tuple(bits(t).clone() for t in mb.rms_norm_fp8(x, None, r, residual_out=h))))
    same(*both(lambda: tuple(bits(t) for t in mb.rms_norm_fp8(x[0, 0:1]))))
    g = grad_inputs(7, 130, "bf16", "bf16", 2)
    for kw in (dict(), dict(weight=g["w"]), dict(weight=g["w"], dh=g["dh"]), dict(dh=g["dh"], dx_dtype=torch.float32)):
        def call():
            d = mb.rms_norm_bwd(g["dy"], g["h"], g["rstd"], **kw)
            assert list(d) == ["dx", "dweight"] + (["dresidual"] if "dh" in kw else [])
            assert "dh" not in kw or (d["dresidual"] is d["dx"]) == ("dx_dtype" not in kw)
            return tuple(d.values())
        same(*both(call))
    q, s = mb.quantize_fp8(x)
    c = torch.empty(7, 7, device="cuda:0")
    same(*both(lambda: (mb.matmul_fp8(q, s, q, s, out=c).clone(),)))
    same(*both(lambda: (mb.matmul_fp8(q[None], s[None], q, s),)))
    lg, nz = logits_of(5, 100, "f32", 3)
    t, k = torch.ones(5, device="cuda:0"), torch.ones(5, dtype=torch.int32, device="cuda:0")
    same(*both(lambda: (mb.sample(lg, nz),)))
    same(*both(lambda: mb.sample(lg, nz, temperature=t, top_k=k, top_p=t, min_p=t * 0, return_prob=True)))
    same(*both(lambda: (mb.sample(lg, nz, top_k=-3),), taken=False))
    for bad in (lambda: mb.rms_norm_fwd(x, w[:5].contiguous()), lambda: mb.rms_norm_fwd(x.t()), lambda: mb.rms_norm_fwd(x, w, r[:3]),
                lambda: mb.rms_norm_fwd(x, w.bfloat16()), lambda: mb.rms_norm_fwd(x, residual_out=h), lambda: mb.rms_norm_fwd(x.double()),
                lambda: mb.rms_norm_fwd(x, w, r, residual_out=x), lambda: mb.rms_norm_fwd(x, eps=-1.0), lambda: mb.rms_norm_fwd(x, out=x),
                lambda: mb.rms_norm_bwd(g["dy"], g["h"], g["rstd"][:3]), lambda: mb.rms_norm_bwd(g["dy"], g["h"], g["rstd"], dh=r),
                lambda: mb.quantize_fp8(x[0]), lambda: mb.quantize_fp8(x.half()), lambda: mb.matmul_fp8(q, s, q[:, :100], s),
                lambda: mb.matmul_fp8(q, s[:3], q, s), lambda: mb.matmul_fp8(x, s, q, s), lambda: mb.matmul_fp8(q, s, q, s, out_dtype=torch.half),
                lambda: mb.matmul_fp8(q[None].expand(2, 7, 130).contiguous(), s[None].expand(2, 7, 2).contiguous(),
                                      q[None].expand(3, 7, 130).contiguous(), s[None].expand(3, 7, 2).contiguous()),
                lambda: mb.sample(lg, nz[:2]), lambda: mb.sample(lg, nz, top_k=t), lambda: mb.sample(lg, nz, temperature=k)):
        with pytest.raises(mb.MBScanError):
            bad()


@pytest.mark.parametrize("V", [256, 1000, 6000, 30000, 60000])
@pytest.mark.parametrize("kind", ["equal", "random", "coarse"])
def test_sample_many_rows(V, kind):
    """200 copies of a sequence draw the same token, call after call, whatever the filters."""
    import paper_2401_13660_amd as mb
    announce(f"sample of 200 rows alike, {V} {kind}")
    for dtype in (torch.float32, torch.bfloat16):
        lg, nz = logits_of(1, V, "f32", 5)
        lg = torch.zeros_like(lg) if kind == "equal" else lg if kind == "random" else (lg * 2).round()
        rows, noise = lg.to(dtype).expand(200, V).contiguous(), nz.expand(200, V).contiguous()
        for kw in (dict(top_k=2), dict(top_k=37), dict(top_k=V - 1), dict(top_p=0.3), dict(top_p=0.999), dict(top_k=V // 2, top_p=0.9),
                   dict(top_k=V // 3, top_p=0.9999999, min_p=1e-3)):
            t, p = mb.sample(rows, noise, return_prob=True, **kw)
            u, r = mb.sample(rows, noise, return_prob=True, **kw)
            assert (t == t[0]).all() and (p == p[0]).all() and torch.equal(t, u) and torch.equal(p, r), (dtype, kw)


def test_a_step_of_a_model():
    """The operators as they follow each other: embedding, then per block the norm in 8 bits, the input projection to (batch, channels, time),
    convolution and scan, their output turned to 8 bits and projected back; the last norm, the logits' product, and the draw."""
    import paper_2401_13660_amd as mb
    announce("a step of a model in 8 bits")
    g = torch.Generator(device="cuda:0").manual_seed(0)
    b, L, width, N, V = 2, 48, 128, 16, 256
    D = 2 * width

    def weight(*shape):
        return torch.randn(shape, generator=g, device="cuda:0") / shape[-1] ** 0.5
    table, tokens = weight(V, width), torch.randint(0, V, (b, L), generator=g, device="cuda:0").to(torch.uint8)
    blocks = [dict(norm=torch.ones(width, device="cuda:0"), w_in=weight(2 * D, width), w_x=weight(8 + 2 * N, D), w_dt=weight(D, 8), w_out=weight(width, D),
                   taps=weight(D, 4), A=-torch.arange(1, N + 1, device="cuda:0").float().repeat(D, 1)) for _ in range(2)]

    def run(project, norm):
        stream, x = mb.embedding_fwd(tokens, table, scale=width ** 0.5), None
        for k in blocks:
            h, stream = norm(x, stream, k["norm"])
            xz = project(h, k["w_in"], "turned")                                                # (b, 2 D, L)
            u, z = xz[:, :D].contiguous(), xz[:, D:].contiguous()
            u = mb.conv1d(u, k["taps"])
            dbc = u.transpose(1, 2) @ k["w_x"].t()
            delta = (dbc[..., :8] @ k["w_dt"].t()).transpose(1, 2).contiguous()
            Bm, C = dbc[..., 8:].transpose(1, 2).chunk(2, 1)
            y = mb.scan_fwd(u, delta, k["A"], Bm.contiguous(), C.contiguous(), z=z)
            x = project(y, k["w_out"], "back")                                                  # (b, L, width)
        h, stream = norm(x, stream, blocks[0]["norm"])
        return project(h, table, "rows")

    def norm8(x, stream, w):
        if x is None:
            return mb.rms_norm_fp8(stream, w), stream
        q, s, h = mb.rms_norm_fp8(x, w, stream)
        return (q, s), h

    def project8(h, w, how):
        wq = mb.quantize_fp8(w, tile=True)
        if how == "turned":
            return mb.matmul_fp8(*wq, *h, out_dtype=torch.float32)
        q, s = mb.quantize_fp8(h, transpose=True) if how == "back" else h
        return mb.matmul_fp8(q.view(b * L, -1), s.view(b * L, -1), *wq, out_dtype=torch.float32).view(b, L, -1)

    def norm64(x, stream, w):
        stream = stream if x is None else stream + x
        return stream / torch.sqrt(stream.square().mean(-1, keepdim=True) + 1e-5) * w, stream

    def project32(h, w, how):
        y = h.transpose(1, 2) @ w.t() if how == "back" else h @ w.t()
        return y.transpose(1, 2).contiguous() if how == "turned" else y
    eight, plain = run(project8, norm8), run(project32, norm64)
    # 8-bit values are within half a step, 2^-4, of their own; independent errors of seven products in a row
    assert (eight - plain).norm() <= 7 * 2.0 ** -4 * plain.norm()
    noise = torch.empty(b, V, device="cuda:0").exponential_(generator=g)
    last = eight[:, -1].contiguous()
    token, prob = mb.sample(last, noise, temperature=0.8, top_k=50, top_p=0.98, return_prob=True)
    for i in range(b):
        t, p, margin = B.sample(np64(last[i]), np64(noise[i]), float(torch.tensor(0.8)), 50, float(torch.tensor(0.98)))
        assert margin < 2e-5 or int(token[i]) == t


def test_training_step():
    """The differentiable operations together: gradients of a projection behind a norm, against torch's of the unrounded one."""
    import paper_2401_13660_amd as mb
    announce("norm and projection in 8 bits, their gradients")
    x, r = randn((3, 50, 96), 1, "f32").requires_grad_(), randn((3, 50, 96), 2, "f32").requires_grad_()
    n, w = torch.ones(96, device="cuda:0", requires_grad=True), (randn((64, 96), 3, "f32") / 10).requires_grad_()
    cy, ch = randn((3, 50, 64), 4, "f32"), randn((3, 50, 96), 5, "f32")
    leaves = (x, r, n, w)
    y, h = mb.rms_norm(x, n, r)
    ((mb.linear_fp8(y, w) * cy).sum() + (h * ch).sum()).backward()
    got = [t.grad.clone() for t in leaves]
    for t in leaves:
        t.grad = None
    h = x + r
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * n
    ((y @ w.t() * cy).sum() + (h * ch).sum()).backward()
    for a, t in zip(got, leaves):
        assert (a - t.grad).norm() <= 2 * 2.0 ** -4 * 1.1 * t.grad.norm()


def test_training_step_in_a_graph():
    """Forward and gradients of the norm and the projection, captured, replayed on new inputs, against eager passes."""
    import paper_2401_13660_amd as mb
    announce("norm and projection in 8 bits: gradients in a graph")
    x, r, cy, ch = (randn((2, 300, 256), k, "bf16") for k in (1, 2, 3, 4))
    w, p = randn((256,), 5, "f32"), randn((384, 256), 6, "f32") / 16
    c = randn((2, 300, 384), 7, "bf16")
    leaves = [x.requires_grad_(), r.requires_grad_(), w.requires_grad_(), p.requires_grad_()]

    def step():
        y, h = mb.rms_norm(x, w, r)
        return torch.autograd.grad([mb.linear_fp8(y, p), y, h], leaves, [c, cy, ch])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        with torch.no_grad():
            x.copy_(randn(x.shape, 10 + k, "bf16"))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b), f"replay {k}"


def test_example_completes():
    """The example's byte-by-byte continuation: bytes, the same for the same seed, and the model's largest logit at temperature 0."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import byte_model as E
    announce("byte model: bytes one by one")
    torch.manual_seed(0)
    model = E.ByteModel(32, 2)
    prompt = torch.randint(0, 256, (3, 20), device="cuda:0").to(torch.uint8)
    a = E.complete(model, prompt, 6)
    assert a.shape == (3, 6) and torch.equal(a, E.complete(model, prompt, 6)) and a.min() >= 0 and a.max() < 256
    with torch.no_grad():
        assert torch.equal(E.complete(model, prompt, 1, temperature=0.0)[:, 0].long(), model.extend(prompt, model.empty(3))[0][:, -1].argmax(1))

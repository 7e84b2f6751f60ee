"""The native entry points of the operators around the layers against the binding's Python code: the same bits, and
what they do not take goes to Python."""
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_clip import tensors
from test_gpu_conv_bwd import inputs
from test_gpu_embedding import randn
from test_gpu_fastcall import both, watched  # noqa: F401  (fixtures)
from test_gpu_verify_sample import case

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def same(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        if x is None or y is None:
            assert x is y
            continue
        assert x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and torch.equal(x, y)


@pytest.mark.parametrize("tok", [torch.uint8, torch.int32, torch.int64])
@pytest.mark.parametrize("opts", [{}, dict(scale=2), dict(out_dtype=torch.float32), dict(scale=0.5, out="given")])
@pytest.mark.parametrize("shape", [(), (7,), (2, 3), (2, 1, 2, 3, 2, 2)])
def test_embedding(both, tok, opts, shape):  # noqa: F811
    import paper_2401_13660_amd as mb
    announce(f"native embedding {tok} {opts} {shape}")
    t = torch.arange(max(1, torch.Size(shape).numel()), device="cuda:0").reshape(shape).to(tok)
    W = randn((48, 24), 1, "bf16")
    kw = dict(opts)
    if "out" in kw:
        kw["out"] = torch.empty(shape + (24,), device="cuda:0")
    same(*both(lambda: mb.embedding_fwd(t, W, **kw).clone()))
    same(*both(lambda: mb.embedding_fwd(t, torch.nn.Parameter(W), **kw).clone()))
    dy = randn(shape + (24,), 2, "bf16")
    kw = dict(opts)
    if "out" in kw:
        kw["out"] = torch.empty(48, 24, device="cuda:0").bfloat16()
    same(*both(lambda: mb.embedding_bwd(t, dy, 48, **kw).clone()))


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("state", [True, False])
def test_conv_bwd(both, bias, state):  # noqa: F811
    import paper_2401_13660_amd as mb
    announce("native conv1d_bwd")
    a = inputs(2, 6, 50, 4, "bf16", "bf16", 3, state)

    def call():
        g = mb.conv1d_bwd(a["x"], a["w"], a["dy"], a["bias"] if bias else None, a["state"], a["dstate_out"])
        assert list(g) == ["dx", "dw", "dbias", "dstate"]
        return tuple(g.values())
    same(*both(call))


def test_norm_and_clip(both):  # noqa: F811
    import paper_2401_13660_amd as mb
    announce("native grad_norm and clip_grad_norm")
    g = tensors([5, 0, 3000, 77], ["f32", "bf16", "bf16", "f32"], 4)
    out = [torch.empty_like(t) for t in g]
    same(*both(lambda: mb.grad_norm(g)))
    same(*both(lambda: mb.grad_norm(tuple(torch.nn.Parameter(t) for t in g))))
    same(*both(lambda: (mb.clip_grad_norm(g, 1, out=out),) + tuple(o.clone() for o in out)))
    same(*both(lambda: (mb.clip_grad_norm(h := [t.clone() for t in g], 0.5),) + tuple(h)))
    same(*both(lambda: mb.grad_norm(t for t in g), taken=False))
    same(*both(lambda: mb.grad_norm(g[2]), taken=False))
    same(*both(lambda: mb.clip_grad_norm([t.clone() for t in g], torch.tensor(0.5)), taken=False))


@pytest.mark.parametrize("V", [256, 2000])
@pytest.mark.parametrize("drafter", ["logits", None])
@pytest.mark.parametrize("probs", [True, False])
def test_verify_sample(both, V, drafter, probs):  # noqa: F811
    import paper_2401_13660_amd as mb
    announce("native verify_sample")
    a = case(4, 3, V, drafter=drafter, ragged=probs, seed=5)
    same(*both(lambda: mb.verify_sample(a["logits"], a["draft"], a["uniform"], a["noise"], a["draft_logits"],
                                        lengths=a["lengths"], temperature=a["temperature"], return_probs=probs)))


def test_declined_calls_end_in_the_same_errors(watched, monkeypatch):  # noqa: F811
    import paper_2401_13660_amd as mb
    from paper_2401_13660_amd import _binding
    announce("native entry points: refusals")
    f, t = torch.ones(4, 6, device="cuda:0"), torch.zeros(4, dtype=torch.int32, device="cuda:0")
    a = case(2, 2, 16, seed=6)
    calls = [lambda: mb.embedding_fwd(t, f.t()), lambda: mb.embedding_fwd(t.short(), f), lambda: mb.embedding_fwd(t, f, out=f),
             lambda: mb.embedding_bwd(t, f, -1), lambda: mb.embedding_bwd(t[:3], f, 4), lambda: mb.grad_norm([]),
             lambda: mb.grad_norm([f, f.t()]), lambda: mb.grad_norm([f.double()]), lambda: mb.clip_grad_norm([f, f], 1.0),
             lambda: mb.clip_grad_norm([f], 1.0, out=[f]), lambda: mb.clip_grad_norm([f], 1.0, out=[f[0]]),
             lambda: mb.clip_grad_norm([f], -1.0), lambda: mb.conv1d_bwd(f, f, f),
             lambda: mb.conv1d_bwd(f[None], f, f[None]),
             lambda: mb.verify_sample(a["logits"], a["draft"].long(), a["uniform"], a["noise"]),
             lambda: mb.verify_sample(a["logits"], a["draft"], a["uniform"], a["noise"], temperature=-1.0)]
    for i, call in enumerate(calls):
        said = []
        for native in (True, False):
            with monkeypatch.context() as m:
                if not native:
                    m.setattr(_binding, "_fast", None)
                with pytest.raises(mb.MBScanError) as e:
                    call()
                said.append(str(e.value))
        assert said[0] == said[1], i

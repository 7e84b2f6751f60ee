"""Tensors that an operator around the layers writes in place are seen as changed: a gradient that was saved before and
is taken after raises, as with torch's own operations, instead of coming out of the new values."""
import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.fixture(params=[True, False], ids=["native", "python"])
def native(request, monkeypatch):
    from paper_2401_13660_amd import _binding
    _binding.load_library()
    if not request.param:
        monkeypatch.setattr(_binding, "_fast", None)
    announce(f"tensors written in place, native {request.param}")


def ones(*shape):
    return torch.ones(*shape, device="cuda:0")


def calls():
    """What is written, and the call that writes it."""
    import paper_2401_13660_amd as mb
    tokens = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    g, h, o, e, w = ones(8), ones(3), ones(8), ones(4, 8), ones(5, 8)
    yield [g, h], lambda: mb.clip_grad_norm([g, h], 0.1)
    yield [o], lambda: mb.clip_grad_norm([g], 0.1, out=[o])
    yield [e], lambda: mb.embedding_fwd(tokens, ones(5, 8), out=e)
    yield [w], lambda: mb.embedding_bwd(tokens, ones(4, 8), 5, out=w)


@pytest.mark.parametrize("which", range(4))
def test_a_saved_tensor_that_changed_raises(native, which):
    written, call = list(calls())[which]
    for t in written:
        x = torch.ones_like(t, requires_grad=True)
        y = (x * t).sum()                                   # saves t for x's gradient
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


def test_views_and_what_is_only_read(native):
    import paper_2401_13660_amd as mb
    flat, g, o = ones(20), ones(4), ones(4)
    versions = flat._version, g._version
    mb.clip_grad_norm([flat[:8], flat[8:]], 0.1)
    assert flat._version > versions[0]                      # written through its views
    mb.clip_grad_norm([g], 0.1, out=[o])
    mb.grad_norm([g, o])
    assert g._version == versions[1]
    version = o._version
    with pytest.raises(mb.MBScanError):
        mb.clip_grad_norm([o], -1.0)
    assert o._version == version


def test_in_inference_mode(native):
    """Tensors made there have no count of their changes."""
    import paper_2401_13660_amd as mb
    g = ones(6)
    with torch.inference_mode():
        h = ones(6)
        mb.clip_grad_norm([g, h], 0.1)
        mb.embedding_fwd(torch.zeros(2, dtype=torch.int32, device="cuda:0"), ones(3, 6), out=torch.empty(2, 6, device="cuda:0"))
    mb.clip_grad_norm([h], 0.05)
    assert abs(float(h.norm()) - 0.05) < 1e-6

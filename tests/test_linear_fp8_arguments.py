"""What the differentiable projection in 8 bits takes and refuses: x of any strides, the same result and gradients as of its copy; a weight is a matrix."""
import pytest
import torch

import paper_2401_13660_amd as mb
from gpu_util import announce, has_gpu


@pytest.mark.parametrize("x,weight,what", [
    ((4, 8), (3, 1, 8), "weight must be"), ((4, 8), (8,), "weight must be"), ((4, 8), None, "weight must be"),
    ((), (3, 8), "x must be"), (None, (3, 8), "x must be"),
])
def test_refusals(x, weight, what):
    a, b = (None if s is None else torch.zeros(s) for s in (x, weight))
    with pytest.raises(mb.MBScanError, match=what):
        mb.linear_fp8(a, b)


STRIDED = {"turned": lambda t: t.t(), "turned in a batch": lambda t: t.view(3, 20, 40).transpose(1, 2), "every other row": lambda t: t[::2],
           "columns cut out": lambda t: t[:, 3:40], "one row for all": lambda t: t[:1].expand(7, 40),
           "one matrix for all": lambda t: t[None].expand(2, 60, 40)}


@pytest.mark.gpu
@pytest.mark.skipif(not has_gpu(), reason="needs a GPU")
@pytest.mark.parametrize("how", STRIDED)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(how, dtype):
    announce(f"linear_fp8 of rows {how} {dtype}")
    g = torch.Generator(device="cuda:0").manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, generator=g, device="cuda:0")
    strided = STRIDED[how](draw(60, 40).to(dtype))
    w = draw(strided.shape[-1], 24).t()                         # (24, k), turned
    dy = draw(24, *strided.shape[:-1]).movedim(0, -1).to(dtype)
    assert not strided.is_contiguous() and not w.is_contiguous() and not dy.is_contiguous()
    got = []
    for a, b, c in ((strided, w, dy), (strided.contiguous(), w.contiguous(), dy.contiguous())):
        a, b = a.detach().requires_grad_(), b.detach().requires_grad_()
        y = mb.linear_fp8(a, b)
        got.append((y.detach(), *torch.autograd.grad(y, (a, b), c)))
    for a, b in zip(*got):
        assert a.shape == b.shape and torch.equal(a, b)

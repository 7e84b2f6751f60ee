"""The convolution's gradient of one sequence, whose rows have a channel's sums whole, and of none.  Tolerances as in
test_gpu_conv_bwd."""
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_conv_bwd import call, check, inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("D,L", [(5, 1), (7, 3), (64, 16), (9, 130), (6, 200), (3, 300), (11, 512), (4, 513), (4500, 530), (4200, 1030), (2, 2048), (2, 2049), (1024, 1100), (3, 5000)])
def test_sequence(K, dtype, out, D, L):
    announce(f"conv1d_bwd (1, {D}, {L}) K={K} {dtype} {out}")
    check(inputs(1, D, L, K, dtype, out, K + D + L))


@pytest.mark.parametrize("shape", [(1, 6, 0), (0, 6, 20), (0, 6, 0)])
def test_nothing(shape):
    """No timestep, or no sequence: dw and dbias are zeros."""
    announce(f"conv1d_bwd {shape}")
    a = inputs(*shape, 4, "f32", "f32", 1)
    for _ in range(4):
        torch.full((64,), 7.0, device="cuda:0")             # the outputs' memory holds no zeros by chance
    g = call(a)
    torch.cuda.synchronize()
    assert (g["dw"] == 0).all() and (g["dbias"] == 0).all()


def test_without_a_bias():
    announce("conv1d_bwd of one sequence without a bias")
    a = inputs(1, 70, 90, 4, "bf16", "f32", 2)
    with_bias = dict(a, bias=torch.zeros(70, device="cuda:0"))
    a["bias"] = None
    g, ref = call(a), call(with_bias)
    torch.cuda.synchronize()
    assert g["dbias"] is None and torch.equal(g["dw"], ref["dw"]) and torch.equal(g["dx"], ref["dx"])

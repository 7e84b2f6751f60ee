"""The convolution's gradient on more than 2^31 elements in whole numbers: every partial sum is exact in fp32, so the sums
over batch and time have to equal the integers', channel by channel, before and past the 32-bit offsets."""
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_large_offsets import DEV, PAST, free_memory  # noqa: F401  (a fixture)

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def whole(n, seed):
    """Integers in -3 .. 3 in bf16: a short random tensor repeated, each time shifted."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    part = torch.randint(-3, 4, (1 << 20,), generator=g, device=DEV).bfloat16()
    out = torch.empty(n, dtype=torch.bfloat16, device=DEV)
    for i, at in enumerate(range(0, n, 1 << 20)):
        m = min(1 << 20, n - at)
        out[at:at + m] = torch.roll(part, i * 97)[:m]
    return out


def test_conv_bwd():
    import paper_2401_13660_amd as mb
    B, D, L = 5, 13001, 33100
    assert B * D * L > PAST and 9 * B * L < 2 ** 24
    announce(f"conv1d_bwd exact ({B}, {D}, {L}): {B * D * L} elements")
    x, dy = whole(B * D * L, 1).view(B, D, L), whole(B * D * L, 2).view(B, D, L)
    w = torch.randint(-2, 3, (D, 4), device=DEV) * 0.5
    g = mb.conv1d_bwd(x, w, dy, torch.zeros(D, device=DEV), apply_silu=False)
    dw, dbias = torch.zeros(D, 4, device=DEV), torch.zeros(D, device=DEV)
    for b in range(B):
        dbias += dy[b].sum(1, dtype=torch.float32)
        for j in range(4):                                  # products within 9 are exact in bf16, their sums in fp32
            back = 3 - j
            dw[:, j] += (dy[b, :, back:] * x[b, :, :L - back]).sum(1, dtype=torch.float32)
    assert dw.abs().max() > 1000
    for k, ref in (("dw", dw), ("dbias", dbias)):
        wrong = (g[k] != ref).reshape(D, -1).any(1).nonzero().flatten().tolist()
        assert not wrong, f"{k}: channels {wrong[:8]} of {len(wrong)}"

"""The rounding of the convolution's weight gradients over long rows.

dw and dbias add a row's products by span (8 terms in a lane here), then the tiles of a row (L / 512), the lanes (6
additions), then stretches and sequences: with T tiles a result is within (8 + T + 6 + 1) 2^-24 of the sum of its terms'
magnitudes.  One running sum per lane over the row would be allowed 8 T.

The terms are all 1 + e with e such that a running sum of n of them, once past n / 2, loses nearly half of its last bit
with every term: n / 4 times 2^-24 in all, which is above the bound."""
import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("L", [32768, 65536])
def test_sums_of_one_stretch(L):
    import paper_2401_13660_amd as mb
    D = 4096                                                # as many rows as leave each in one stretch
    announce(f"conv1d_bwd (1, {D}, {L}): the rounding of dw and dbias")
    n, tiles = L // 64, L // 512
    c = 1.0 + 0.499 * 2.0 ** -24 * n                        # half of the last bit of n / 2 .. n is 2^-25 n
    x = torch.full((1, D, L), c, device="cuda:0")
    dy = torch.ones(1, D, L, dtype=torch.bfloat16, device="cuda:0")
    g = mb.conv1d_bwd(x, torch.zeros(D, 4, device="cuda:0"), dy, torch.zeros(D, device="cuda:0"), apply_silu=False)
    term = x[0, 0, 0].double().item()
    terms = torch.arange(L - 3, L + 1, device="cuda:0", dtype=torch.float64)
    err = (g["dw"].double() / (terms * term) - 1).abs().max().item()
    assert err <= (8 + tiles + 6 + 1) * 2.0 ** -24, f"{err:.2e}"
    assert (g["dbias"] == L).all()

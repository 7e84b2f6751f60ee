"""The gradient of a table that no token names, of any width: zeros."""
import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("V,d", [(1, 1), (3, 524288), (1, 524289), (1, 2000001), (5, 3000000), (1, (1 << 34) - 4), (1, (1 << 34) + 3)])
def test_zeros(V, d):
    import paper_2401_13660_amd as mb
    announce(f"embedding_bwd of no tokens, {V} rows of {d}")
    torch.cuda.empty_cache()
    out = torch.ones(V, d, dtype=torch.bfloat16, device="cuda:0")
    tokens = torch.zeros(0, dtype=torch.int32, device="cuda:0")
    mb.embedding_bwd(tokens, torch.zeros(0, d, dtype=torch.bfloat16, device="cuda:0"), V, out=out)
    for part in out.view(-1).split(1 << 30):
        assert not part.any()
    del out, part
    torch.cuda.empty_cache()

"""The embedding's gradient of as many tokens as its contract allows and the card's memory leaves time for: more groups of
sorted tokens than 2^22.  Whole numbers, so the sums are exact in fp32."""
import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def test_a_billion_bytes():
    import paper_2401_13660_amd as mb
    n = (1 << 30) + 77
    announce(f"embedding_bwd of {n} bytes, one column")
    torch.cuda.empty_cache()
    g = torch.Generator(device="cuda:0").manual_seed(1)
    tokens = torch.randint(0, 256, (n,), generator=g, device="cuda:0", dtype=torch.uint8)
    tokens[: 1 << 20] = 7                                   # a longer run than the others
    dy = torch.randint(0, 2, (n,), generator=g, device="cuda:0", dtype=torch.uint8)
    got = mb.embedding_bwd(tokens, dy.bfloat16()[:, None], 256)
    ref = torch.zeros(256, dtype=torch.int64, device="cuda:0")
    for t, d in zip(tokens.split(1 << 27), dy.split(1 << 27)):
        ref += torch.bincount(t[d == 1], minlength=256)
    assert ref.max() < 1 << 24 and torch.equal(got[:, 0].long(), ref)
    del tokens, dy
    torch.cuda.empty_cache()

"""The operators around the layers on tensors of more than 2^31 elements: what lies past the 32-bit offsets is compared
with the same operator on that part alone (the same bits where the sums are the same), or with a plain sum."""
import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
DEV = "cuda:0"
PAST = 2 ** 31


@pytest.fixture(autouse=True)
def free_memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def noise(n, dtype=torch.bfloat16):
    """Values in [-1, 1) that cost little to make: a short random tensor repeated, each time shifted."""
    part = torch.rand(1 << 20, device=DEV).mul_(2).sub_(1).to(dtype)
    out = torch.empty(n, dtype=dtype, device=DEV)
    for i, at in enumerate(range(0, n, 1 << 20)):
        m = min(1 << 20, n - at)
        out[at:at + m] = torch.roll(part, i * 97)[:m]
    return out


def test_embedding():
    import paper_2401_13660_amd as mb
    d, n = 2304, (1 << 20) + 1000
    assert n * d > PAST
    announce(f"embedding of {n} tokens, width {d}: {n * d} elements")
    tokens = torch.randint(0, 256, (n,), device=DEV, dtype=torch.uint8)
    W = torch.randn(256, d, device=DEV).bfloat16()
    y = mb.embedding_fwd(tokens, W, scale=2.0)
    for at in (0, n // 2, PAST // d - 1, PAST // d + 1, n - 50):
        assert torch.equal(y[at:at + 50], mb.embedding_fwd(tokens[at:at + 50].contiguous(), W, scale=2.0))
    g = mb.embedding_bwd(tokens, y, 256)
    # the rows of y are those of the table, so the sums are counts times rows, up to fp32's rounding of the sums
    counts = torch.bincount(tokens.long(), minlength=256).double()
    ref = counts[:, None] * (2.0 * W.double()).bfloat16().double()
    assert ((g.double() - ref).abs() <= (counts[:, None] + 2) * 2.0 ** -24 * ref.abs()).all()


def test_conv_bwd():
    import paper_2401_13660_amd as mb
    B, D, L = 5, 13001, 33100
    assert B * D * L > PAST
    announce(f"conv1d_bwd ({B}, {D}, {L}): {B * D * L} elements")
    x, dy = noise(B * D * L).view(B, D, L), noise(B * D * L).view(B, D, L)
    w, bias = torch.rand(D, 4, device=DEV) - 0.5, torch.rand(D, device=DEV) - 0.5
    g = mb.conv1d_bwd(x, w, dy, bias)
    for b, d in ((0, 0), (2, 7000), (4, 12000), (4, D - 1)):
        s = mb.conv1d_bwd(x[b:b + 1, d:d + 1].contiguous(), w[d:d + 1].contiguous(), dy[b:b + 1, d:d + 1].contiguous(),
                          bias[d:d + 1].contiguous())
        assert torch.equal(g["dx"][b, d], s["dx"][0, 0]), (b, d)
    d = D - 1
    s = mb.conv1d_bwd(x[:, d:].contiguous(), w[d:].contiguous(), dy[:, d:].contiguous(), bias[d:].contiguous())
    mag = (x[:, d].float().abs().max() * dy[:, d].float().abs()).sum()
    assert ((g["dw"][d] - s["dw"][0]).abs() <= 2 * B * L * 2.0 ** -24 * mag).all()


def test_clip():
    import paper_2401_13660_amd as mb
    n = PAST + 12345
    announce(f"clip_grad_norm of one tensor of {n} elements and a small one")
    g, h = noise(n), torch.randn(1000, device=DEV)
    was, hwas = g.clone(), h.clone()
    ref = (sum(float(c.double().square().sum()) for c in g.split(1 << 28)) + float(h.double().square().sum())) ** 0.5
    norm = mb.clip_grad_norm([g, h], 0.5 * ref)
    assert abs(float(norm) - ref) <= 2 * 2.0 ** -24 * ref
    factor = 0.5 * ref / (ref + 1e-6)
    for at in (0, n // 2, PAST - 500, PAST + 1, n - 1000):
        r = was[at:at + 1000].double() * factor
        assert ((g[at:at + 1000].double() - r).abs() <= 2.0 ** -8 * r.abs()).all()
    assert ((h.double() - hwas.double() * factor).abs() <= 2.0 ** -21 * hwas.double().abs()).all()


@pytest.mark.parametrize("V,B,n", [(300, 1800000, 3), (40000, 9000, 5)])
def test_verify_sample(V, B, n):
    import paper_2401_13660_amd as mb
    assert B * (n + 1) * V > PAST
    announce(f"verify_sample ({B}, {n}, {V}): {B * (n + 1) * V} logits")
    logits = noise(B * (n + 1) * V).view(B, n + 1, V)
    draft = torch.randint(0, V, (B, n), device=DEV, dtype=torch.int32)
    uniform, e = torch.rand(B, n, device=DEV) * 0.01, torch.empty(B, V, device=DEV).exponential_()
    got = mb.verify_sample(logits, draft, uniform, e, return_probs=True)
    for at in (0, B // 2, PAST // ((n + 1) * V) + 1, B - 40):
        part = [t[at:at + 40].contiguous() for t in (logits, draft, uniform, e)]
        for x, y in zip(got, mb.verify_sample(*part, return_probs=True)):
            assert torch.equal(x[at:at + 40], y)

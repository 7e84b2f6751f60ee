"""The embedding's gradient at the edges between its ways of adding up: a workgroup per row or per token (few tokens), the
sort by one workgroup, the sort by many.  Tolerances as in test_gpu_embedding."""
import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_embedding import DT, TOK, check_bwd, randn, shifted

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
FEW, MANY, TOO_MANY = 200, 9000, 131073        # rows of a table: a workgroup each; a workgroup per token; sorted


def text(n, V, seed, padding=True):
    """Tokens of which some are common, most rare and a few padding or past the table."""
    r = np.random.default_rng(seed)
    t = np.minimum(r.geometric(min(1.0, 9 / V), n) - 1, V - 1)
    t[r.random(n) < 0.2] = V // 2
    if padding:
        t[r.random(n) < 0.1] = -1
        t[r.random(n) < 0.05] = V
    return torch.from_numpy(t).to("cuda:0")


@pytest.mark.parametrize("V", [FEW, MANY, TOO_MANY])
@pytest.mark.parametrize("n", [0, 1, 2, 7, 8, 9, 63, 64, 65, 511, 512, 513, 520, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097])
def test_tokens(n, V):
    announce(f"embedding_bwd n={n} V={V}")
    check_bwd(text(n, V, n).int(), randn((n, 36), n + 1, "bf16"), V, 1.5, "f32")


@pytest.mark.parametrize("dd,od", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("d", [1, 2, 3, 4, 5, 8, 9, 255, 256, 257, 260, 511, 513, 1792])
def test_widths(d, dd, od):
    announce(f"embedding_bwd dim={d} {dd}->{od}")
    for V in (FEW, MANY) if d > 257 else (FEW, MANY, TOO_MANY):
        check_bwd(text(700, V, d), randn((700, d), d + 1, dd), V, -0.5, od)


@pytest.mark.parametrize("n,V,d", [(2048, 4096, 256), (2048, 4096, 257), (1024, 5000, 512), (1025, 5000, 512), (1024, 5000, 513),
                                   (700, 1723, 4), (700, 1724, 4), (700, 1725, 4), (1500, 4097, 257), (1500, 2048, 513),
                                   (40, 131072, 5), (2048, 131072, 3), (3, 1, 5), (100, 1025, 700), (100, 2049, 600)])
def test_limits(n, V, d):
    announce(f"embedding_bwd n={n} V={V} dim={d}")
    check_bwd(text(n, V, V + d), randn((n, d), 3, "f32"), V, 1.0, "f32")


@pytest.mark.parametrize("tok,n", [("i32", 2049), ("i64", 3000), ("u8", 4096), ("i32", 4097), ("i64", 5000), ("i32", 32768),
                                   ("u8", 32769), ("i64", 65536), ("i32", 65537)])
@pytest.mark.parametrize("V", [256, 257, 511, 700, 1023, 1024, 1025])
def test_a_few_more_rows_than_bytes(tok, n, V):
    announce(f"embedding_bwd n={n} V={V} {tok}")
    t = text(n, V, n + V, tok != "u8").to(TOK[tok])
    check_bwd(t, randn((n, 12), 5, "bf16"), V, 1.0, "f32")
    check_bwd(t.clamp(max=0), randn((n, 12), 6, "bf16"), V, 1.0, "bf16")


@pytest.mark.parametrize("V", [FEW, MANY, TOO_MANY])
@pytest.mark.parametrize("tok", ["u8", "i32", "i64"])
def test_one_value_and_runs(tok, V):
    """One row takes every token; each wave's share has a token of its own; the last token is another."""
    announce(f"embedding_bwd one value, runs: {tok} V={V}")
    dy = randn((2048, 200), 4, "bf16")
    for t in (torch.full((2048,), 7), torch.arange(2048) // 256, torch.cat([torch.full((2047,), 255), torch.tensor([3])])):
        check_bwd(t.to("cuda:0").to(TOK[tok]), dy, V, 1.0, "f32")


@pytest.mark.parametrize("V", [FEW, MANY, TOO_MANY])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padding_infinities_and_addresses(dtype, V):
    import paper_2401_13660_amd as mb
    announce(f"embedding_bwd padding, infinities, odd addresses: {dtype} V={V}")
    t = text(1001, V, 5)
    dy = randn((1001, 133), 6, dtype)
    t[17], t[18] = 2 ** 40 + 3, -2 ** 63
    out = (t < 0) | (t >= V)
    dy[out] = float("nan")
    dy[t == V // 2] = float("inf")
    g = mb.embedding_bwd(shifted(t, 1), shifted(dy, 1), V, out=shifted(torch.ones(V, 133, dtype=DT[dtype], device="cuda:0"), 3))
    ref = mb.embedding_bwd(t, dy.masked_fill(out[:, None], 0.0), V, out_dtype=DT[dtype])
    torch.cuda.synchronize()
    assert torch.equal(g, ref)
    assert torch.isinf(g[V // 2]).all() and torch.isfinite(g).all(1).sum() == V - 1
    dy[t == V // 2] = 1.0
    check_bwd(t, dy.masked_fill(out[:, None], 0.0), V, 1.0, "f32")


@pytest.mark.parametrize("V", [FEW, MANY, TOO_MANY])
def test_in_a_graph(V):
    """Replays, with other work and other tokens between them."""
    import paper_2401_13660_amd as mb
    announce(f"embedding_bwd in a graph: V={V}")
    t, dy, out = text(600, V, 7, False).int(), randn((600, 64), 8, "bf16"), torch.empty(V, 64, device="cuda:0")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mb.embedding_bwd(t, dy, V, out=out)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mb.embedding_bwd(t, dy, V, out=out)
    for seed in range(9, 13):
        t.copy_(text(600, V, seed, False))
        out.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mb.embedding_bwd(t, dy, V)), seed

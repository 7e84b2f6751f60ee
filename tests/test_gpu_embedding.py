"""GPU parity of the embedding and its gradient against 64 bits.

Tolerances: forward, one fp32 product (2^-24) and, for bf16, one rounding (2^-9): each doubled.  Gradient: a sum of n
fp32 terms in any order is within (n + 2) 2^-24 of the sum of their magnitudes, plus the rounding to bf16."""
import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import model_ops as M

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOK = {"u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}
U = 2.0 ** -24


def shifted(t, by):
    """A dense copy of t that starts `by` elements into its allocation."""
    buf = torch.zeros(t.numel() + by, dtype=t.dtype, device=t.device)
    buf[by:] = t.reshape(-1)
    return buf[by:].view(t.shape)


def randn(shape, seed, dtype):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda:0").to(DT[dtype])


def np64(t):
    return t.double().cpu().numpy()


def check_fwd(tokens, W, scale, out_dtype):
    import paper_2401_13660_amd as mb
    y = mb.embedding_fwd(tokens, W, scale=scale, out_dtype=DT[out_dtype])
    torch.cuda.synchronize()
    assert y.dtype == DT[out_dtype] and y.shape == tokens.shape + (W.shape[1],)
    ref = M.embedding(tokens.cpu().numpy(), np64(W), scale)
    got = np64(y)
    tol = 2 * U if out_dtype == "f32" else 2.0 ** -8
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert (np.abs(got - ref)[~np.isnan(ref)] <= tol * np.abs(ref)[~np.isnan(ref)]).all()


def check_bwd(tokens, dy, V, scale, out_dtype):
    import paper_2401_13660_amd as mb
    g = mb.embedding_bwd(tokens, dy, V, scale=scale, out_dtype=DT[out_dtype])
    again = mb.embedding_bwd(tokens, dy, V, scale=scale, out_dtype=DT[out_dtype])
    torch.cuda.synchronize()
    assert g.dtype == DT[out_dtype] and g.shape == (V, dy.shape[-1])
    assert torch.equal(g, again), "two calls differ"
    t, d64 = tokens.cpu().numpy(), np64(dy)
    ref, mag = M.embedding_grad(t, d64, V, scale), M.embedding_grad(t, np.abs(d64), V, abs(scale))
    n = np.bincount(t.astype(np.int64).ravel()[(t.ravel() >= 0) & (t.ravel() < V)], minlength=V)[:, None]
    tol = (n + 2) * U * mag + (0 if out_dtype == "f32" else 2.0 ** -8) * np.abs(ref)
    bad = np.abs(np64(g) - ref) > tol
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, rows {np.unique(np.nonzero(bad)[0])[:8]}"
    assert (np64(g)[n[:, 0] == 0] == 0).all()


@pytest.mark.parametrize("tok", ["u8", "i32", "i64"])
@pytest.mark.parametrize("wd,od", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (3, 5, 7), (33, 256, 64), (130, 256, 1792), (65, 300, 1001), (17, 70000, 24)])
def test_forward(tok, wd, od, n, V, d):
    announce(f"embedding_fwd n={n} V={V} d={d} {tok} {wd}->{od}")
    r = np.random.default_rng(n + V)
    t = r.integers(0, min(V, 256 if tok == "u8" else V), n)
    check_fwd(torch.from_numpy(t).to("cuda:0").to(TOK[tok]), randn((V, d), 5, wd), 1.5, od)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 37, 256])
def test_forward_padding_mistakes_and_alignment(dtype, d):
    announce(f"embedding_fwd: padding, tokens past the table, odd addresses, {dtype} d={d}")
    t = torch.tensor([[0, -1, 9], [10, 2 ** 40, -2 ** 63], [3, 9, 1 << 31]], device="cuda:0")
    W = randn((10, d), 6, dtype)
    check_fwd(t, W, -0.25, dtype)
    check_fwd(shifted(t, 1), shifted(W, 1), 1.0, dtype)
    check_fwd(t.clamp(-5, 2 ** 31 - 1).int()[:, :2].contiguous(), shifted(W, 3), 1.0, dtype)
    import paper_2401_13660_amd as mb
    out = shifted(torch.zeros(3, 3, d, dtype=DT[dtype], device="cuda:0"), 1)
    assert mb.embedding_fwd(t, W, out=out).data_ptr() == out.data_ptr()
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(out, nan=7.0), torch.nan_to_num(mb.embedding_fwd(t, W), nan=7.0))


def test_forward_infinite_rows():
    """Rows that are not looked up do not touch the others; padding is zero whatever the table holds."""
    import paper_2401_13660_amd as mb
    announce("embedding_fwd: infinities and NaN in the table")
    W = randn((6, 40), 7, "f32")
    W[0] = float("inf")
    W[5] = float("nan")
    y = mb.embedding_fwd(torch.tensor([-1, 2, 0, 5], device="cuda:0"), W, scale=2.0)
    torch.cuda.synchronize()
    assert (y[0] == 0).all() and torch.equal(y[1], 2 * W[2]) and torch.isinf(y[2]).all() and torch.isnan(y[3]).all()


@pytest.mark.parametrize("tok", ["u8", "i32", "i64"])
@pytest.mark.parametrize("dd,od", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,V,d", [(0, 4, 5), (1, 1, 1), (63, 3, 7), (64, 256, 64), (1000, 256, 1792), (2049, 255, 100),
                                   (5000, 257, 33), (3000, 40000, 20), (700, 70001, 9)])
def test_gradient(tok, dd, od, n, V, d):
    announce(f"embedding_bwd n={n} V={V} d={d} {tok} {dd}->{od}")
    r = np.random.default_rng(n + V + d)
    t = np.minimum(r.geometric(min(1.0, 20 / V), n) - 1, V - 1)
    t = t % 256 if tok == "u8" else t
    t = torch.from_numpy(t % V).to("cuda:0").to(TOK[tok])
    check_bwd(t, randn((n, d), 8, dd), V, 1.5, od)


@pytest.mark.parametrize("V,n", [(256, 20000), (1, 4097), (30000, 20000)])
def test_gradient_of_one_token(V, n):
    """Every token the same: one row takes them all."""
    announce(f"embedding_bwd: {n} equal tokens, V={V}")
    t = torch.full((n,), V - 1, dtype=torch.int32, device="cuda:0")
    check_bwd(t, randn((n, 40), 9, "bf16"), V, 1.0, "f32")


def test_gradient_ignores_padding_and_mistakes():
    announce("embedding_bwd: padding and tokens past the table")
    r = np.random.default_rng(10)
    t = r.integers(-3, 14, 999)
    t[::50] = 2 ** 40 + 3
    t[1::50] = -2 ** 63
    tokens = torch.from_numpy(t).to("cuda:0")
    dy = randn((999, 77), 11, "f32")
    dy[(tokens < 0) | (tokens >= 10)] = float("nan")      # what padding carries is not read
    import paper_2401_13660_amd as mb
    g = mb.embedding_bwd(tokens, dy, 10)
    clean = mb.embedding_bwd(tokens, torch.nan_to_num(dy), 10)
    torch.cuda.synchronize()
    assert torch.isfinite(g).all() and torch.equal(g, clean)
    check_bwd(tokens, torch.nan_to_num(dy), 10, 1.0, "f32")
    check_bwd(torch.full_like(tokens, -1), torch.nan_to_num(dy), 10, 1.0, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 515, 520, 2304])
def test_gradient_alignment(dtype, d):
    announce(f"embedding_bwd: odd addresses, {dtype} d={d}")
    t = torch.from_numpy(np.random.default_rng(12).integers(0, 30, (3, 100))).to("cuda:0")
    dy = randn((3, 100, d), 13, dtype)
    check_bwd(shifted(t, 1), shifted(dy, 1), 30, 1.0, "f32")
    import paper_2401_13660_amd as mb
    out = shifted(torch.zeros(30, d, device="cuda:0").to(DT[dtype]), 1)
    mb.embedding_bwd(t, dy, 30, out=out)
    ref = mb.embedding_bwd(t, dy, 30, out_dtype=DT[dtype])
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_autograd_and_differences():
    """The gradient that autograd returns is the slope of the loss (which is linear in the table: a difference over
    a step of 1/2 has only the roundings of its two sums, 2 n d 2^-24 of their magnitudes)."""
    import paper_2401_13660_amd as mb
    announce("embedding: autograd and differences")
    t = torch.from_numpy(np.random.default_rng(14).integers(-1, 12, (4, 25))).to("cuda:0")
    W = randn((12, 6), 15, "f32").requires_grad_()
    dy = randn((4, 25, 6), 16, "f32")
    y = mb.embedding(t, W, scale=3.0)
    y.backward(dy)
    for v, k in ((0, 0), (5, 3), (11, 5)):
        losses = []
        for h in (0.5, -0.5):
            Wh = W.detach().clone()
            Wh[v, k] += h
            losses.append(float((mb.embedding_fwd(t, Wh, scale=3.0).double() * dy.double()).sum()))
        mag = float((y.detach().abs() * dy.abs()).sum()) + 1.0
        assert abs((losses[0] - losses[1]) - float(W.grad[v, k])) <= 2 * 600 * U * mag
    wb = W.detach().bfloat16().requires_grad_()
    mb.embedding(t, wb).sum().backward()
    assert wb.grad.dtype == torch.bfloat16


def test_refusals():
    import paper_2401_13660_amd as mb
    announce("embedding: refusals")
    t = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    W, dy = torch.zeros(5, 8, device="cuda:0"), torch.zeros(4, 8, device="cuda:0")
    for call in (lambda: mb.embedding_fwd(t, W.half()), lambda: mb.embedding_fwd(t.short(), W),
                 lambda: mb.embedding_fwd(t, W.t()), lambda: mb.embedding_fwd(t.cpu(), W),
                 lambda: mb.embedding_fwd(t, W, out=torch.zeros(4, 7, device="cuda:0")),
                 lambda: mb.embedding_bwd(t, dy[:3], 5), lambda: mb.embedding_bwd(t, dy, -1),
                 lambda: mb.embedding_bwd(t, dy.t().contiguous().t(), 5), lambda: mb.embedding_bwd(t, dy, 4, out=dy),
                 lambda: mb.embedding_fwd(torch.zeros(5, dtype=torch.int32, device="cuda:0"), W, out=W)):
        with pytest.raises(mb.MBScanError):
            call()


@pytest.mark.parametrize("n,V", [(6000, 70001), (20000, 20000000), (32768, 3000), (33000, 3000), (40000, 70000), (300001, 400),
                                 (262145, 256), (4096, 300), (4097, 300)])
def test_gradient_of_many_tokens(n, V):
    """The sort in one, two, three and four passes, by one workgroup and by many, that count ahead and that do not."""
    import paper_2401_13660_amd as mb
    d = 3 if V < 10 ** 6 else 1
    announce(f"embedding_bwd n={n} V={V} d={d}")
    r = np.random.default_rng(n + V)
    t = torch.from_numpy(np.where(r.random(n) < 0.3, r.integers(0, 5, n), r.integers(-1, V + 1, n))).to("cuda:0")
    dy = randn((n, d), n, "f32")
    g = mb.embedding_bwd(t, dy, V)
    again = mb.embedding_bwd(t, dy, V)
    ok = (t >= 0) & (t < V)
    ref = torch.zeros(V, d, dtype=torch.float64, device="cuda:0").index_add_(0, t[ok], dy[ok].double())
    mag = torch.zeros(V, d, dtype=torch.float64, device="cuda:0").index_add_(0, t[ok], dy[ok].double().abs())
    count = torch.bincount(t[ok], minlength=V)[:, None]
    assert torch.equal(g, again)
    assert ((g.double() - ref).abs() <= (count + 2) * U * mag).all()

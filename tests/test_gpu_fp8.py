"""GPU parity of matrices in 8 bits and of their products.

Quantising is three fp32 steps and one rounding, each defined: the same bits as the definition's in numpy.  A product of
8-bit values is exact in fp32; a block's sum of 128 of them is taken to be off by a step (2^-23) of the magnitudes' sum
per term at most, the scaling and the blocks' sum by half a step each, and a 16-bit result by half of its own.

For a 16-bit result the matrix unit first sums 8 neighbouring products each, with 14 bits from the largest's leading one
down: beside a product of 2^16, one of 2^3 in the same 8 counts and one of 2^2 does not.  Of such an 8, 7 products lose less than
2^-13 of the largest each.  That largest is at most the largest value of a's 8 times the largest of b's, so 7 x 2^-13 times
the product of the two matrices of such largest values, summed over the eights, bounds what is lost.

Sums of whole numbers of which no 8 spread over 14 bits, and no sum over 24, have no error at all."""
import numpy as np
import pytest
import torch

from gpu_util import announce, has_gpu
from oracle import block_ops as B
from test_gpu_embedding import DT, np64, randn, shifted

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
U = 2.0 ** -24
FP8 = torch.float8_e4m3fn


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def check_quant(x, tile, transpose):
    import paper_2401_13660_amd as mb
    q, s = mb.quantize_fp8(x, tile=tile, transpose=transpose)
    torch.cuda.synchronize()
    flat = x.float().cpu().numpy().reshape((-1,) + tuple(x.shape[-2:]))
    R, C = (x.shape[-1], x.shape[-2]) if transpose else x.shape[-2:]
    assert q.dtype == FP8 and q.shape == x.shape[:-2] + (R, C)
    assert s.shape == x.shape[:-2] + (-(-R // 128) if tile else R, -(-C // 128))
    qc, sc = codes(q).reshape(-1, R, C), s.cpu().numpy().reshape(-1, s.shape[-2], s.shape[-1])
    for i, m in enumerate(flat):
        want, scales = B.quantize(m.T if transpose else m, tile)
        assert np.array_equal(sc[i], scales)
        nan = np.isnan(B.E4M3[want])
        assert np.array_equal(qc[i][~nan], want[~nan]) and np.isnan(B.E4M3[qc[i][nan]]).all()


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("shape", [(1, 1), (1, 300), (300, 1), (7, 16), (128, 128), (129, 127), (130, 261), (5, 1000), (257, 640), (2, 3, 100, 140)])
def test_quantize(shape, tile, transpose):
    announce(f"quantize_fp8 {shape} tile {tile} transpose {transpose}")
    for dtype in ("f32", "bf16"):
        x = (randn(shape, 1, "f32") * torch.exp(randn(shape[:-1] + (1,), 2, "f32"))).to(DT[dtype])
        check_quant(x, tile, transpose)
        check_quant(shifted(x, 3), tile, transpose)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("tile", [False, True])
def test_quantize_extremes(tile, transpose):
    """Zeros, values whose scale is too small to divide by, the type's largest, NaN and infinities."""
    announce("quantize_fp8 of extremes")
    x = randn((260, 260), 4, "f32")
    x[:128, :128] = 0
    x[130:, :100] = 1e-44
    x[:100, 140:] = torch.finfo(torch.float32).max
    x[5, 7] = float("nan")
    x[200, 200] = float("nan")
    check_quant(x, tile, transpose)
    import paper_2401_13660_amd as mb
    x = randn((130, 130), 5, "f32")
    x[3, 5] = float("inf")
    q, s = mb.quantize_fp8(x, tile=tile, transpose=transpose)
    torch.cuda.synchronize()
    assert torch.isinf(s).sum() == 1
    back = q.float() * (s.repeat_interleave(128, 1)[:, :130].repeat_interleave(128, 0)[:130] if tile else s.repeat_interleave(128, 1)[:, :130])
    assert torch.isnan(back).sum() == (128 * 128 if tile else 128)


def test_quantize_every_rounding():
    """Every bf16 value of a few binades around each border of 8 bits, with a largest value that makes the scale 1."""
    import paper_2401_13660_amd as mb
    announce("quantize_fp8 of every bf16 value up to 448")
    bits = torch.arange(0, 0x43e1, dtype=torch.int32)                       # 0 to 448
    v = (bits << 16).view(torch.float32)
    v = torch.cat([v, -v])
    rows = -(-len(v) // 127)
    x = torch.zeros(rows, 128)
    body = torch.zeros(rows * 127)
    body[:len(v)] = v
    x[:, :127] = body.view(rows, 127)
    x[:, 127] = 448.0
    for dtype in ("f32", "bf16"):
        q, s = mb.quantize_fp8(x.to("cuda:0", DT[dtype]))
        torch.cuda.synchronize()
        assert (s == 1).all()
        assert np.array_equal(codes(q), B.to_e4m3(x.double().numpy()))


def test_quantize_nothing_and_past_32_bits():
    import paper_2401_13660_amd as mb
    announce("quantize_fp8 of nothing, and past 2^31 elements")
    for shape in ((0, 5), (5, 0), (0, 3, 4)):
        q, s = mb.quantize_fp8(torch.empty(shape, device="cuda:0"), transpose=True)
        assert q.numel() == 0
    rows, cols = 2048, (1 << 20) + 300
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    x[-130:, -300:] = randn((130, 300), 3, "bf16")
    for transpose in (False, True):
        q, s = mb.quantize_fp8(x, transpose=transpose)
        part = x[-256:, -(300 + (1 << 10)):].contiguous()                  # whole blocks: 2^20 and 2048 are multiples of 128
        sq, ss = mb.quantize_fp8(part, transpose=transpose)
        R, C = sq.shape
        assert torch.equal(q[-R:, -C:].contiguous().view(torch.uint8), sq.view(torch.uint8))
        assert torch.equal(s[-R:, -ss.shape[1]:], ss)
        del q, s


def operand(rows, k, seed, tile, batch=None):
    """Codes and scales as if quantised, without the library: any codes but NaN, any scales."""
    g = torch.Generator().manual_seed(seed)
    lead = () if batch is None else (batch,)
    q = torch.randn(lead + (rows, k), generator=g).mul_(60).to(FP8).to("cuda:0")
    s = torch.rand(lead + (-(-rows // 128) if tile else rows, -(-k // 128)), generator=g).add_(0.1).to("cuda:0")
    return q, s


def values(q, s):
    """fp64 values, (batch, rows, k)."""
    rows, k = q.shape[-2:]
    each = s.double().repeat_interleave(128, -1)[..., :k]
    if s.shape[-2] != rows:
        each = each.repeat_interleave(128, -2)[..., :rows, :]
    v = q.double() * each
    return v if v.dim() == 3 else v[None]


def eights(va, vb):
    """Sums over 8 neighbouring places each of the largest magnitude of a row of va times that of a column of vb."""
    pad = -va.shape[2] % 8
    ta = torch.nn.functional.pad(va.abs(), (0, pad)).unflatten(2, (-1, 8)).amax(3)
    tb = torch.nn.functional.pad(vb.abs(), (0, 0, 0, pad)).unflatten(1, (-1, 8)).amax(2)
    return torch.matmul(ta, tb)


def check_matmul(a, sa, b, sb, out="f32"):
    import paper_2401_13660_amd as mb
    c = mb.matmul_fp8(a, sa, b, sb, out_dtype=DT[out])
    again = mb.matmul_fp8(a, sa, b, sb, out_dtype=DT[out])
    torch.cuda.synchronize()
    m, n, k = a.shape[-2], b.shape[-2], a.shape[-1]
    lead = tuple(a.shape[:-2]) or tuple(b.shape[:-2])
    assert c.shape == lead + (m, n) and c.dtype == DT[out]
    assert torch.equal(c, again), "two calls differ"
    va, vb = values(a, sa), values(b, sb).transpose(1, 2).contiguous()
    ref, size = torch.matmul(va, vb), torch.matmul(va.abs(), vb.abs())
    blocks = -(-k // 128)
    tol = (128 * 2 * U + (blocks + 3) * U) * size
    if out == "bf16":
        tol = tol + 7 * 2.0 ** -13 * eights(va, vb) + 2.0 ** -8 * ref.abs()
    off = (c.double().view(ref.shape) - ref).abs() - tol
    assert (off <= 0).all(), f"{int((off > 0).sum())} of {off.numel()} off, first at {(off > 0).nonzero()[0].tolist()}"


SIZES = [(1, 1, 1), (1, 16, 16), (3, 5, 7), (16, 16, 128), (17, 33, 129), (1, 300, 256), (300, 1, 256), (32, 512, 1792), (64, 64, 64),
         (100, 144, 3584), (127, 129, 127), (128, 128, 128), (129, 257, 272), (200, 1000, 520), (1021, 144, 384), (513, 300, 1003),
         (2, 4000, 1024), (48, 1000, 2304), (700, 700, 144), (1500, 1700, 272), (2900, 1300, 400), (4100, 4100, 272), (8200, 2100, 640),
         (5, 9000, 200), (5, 20000, 130), (9000, 5, 200), (20000, 5, 130), (40, 7168, 256), (30, 17000, 128), (17000, 30, 128), (500, 1000, 1030),
         (700, 900, 260), (60, 40000, 140), (40000, 60, 140), (1300, 1100, 1001)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("a_tile,b_tile", [(False, True), (True, False), (False, False), (True, True)])
def test_matmul(m, n, k, a_tile, b_tile):
    announce(f"matmul_fp8 {m} x {n} x {k} tiles {a_tile} {b_tile}")
    for out in ("f32", "bf16"):
        check_matmul(*operand(m, k, 1, a_tile), *operand(n, k, 2, b_tile), out)


@pytest.mark.parametrize("m,n,k", [(5, 40, 100), (130, 300, 256), (300, 20, 400)])
@pytest.mark.parametrize("ab,bb", [(3, None), (None, 3), (3, 3), (1, None)])
def test_matmul_batches(m, n, k, ab, bb):
    announce(f"matmul_fp8 batches {ab} {bb} of {m} x {n} x {k}")
    check_matmul(*operand(m, k, 3, False, ab), *operand(n, k, 4, True, bb), "bf16")
    check_matmul(*operand(m, k, 3, True, ab), *operand(n, k, 4, False, bb), "f32")


@pytest.mark.parametrize("m,n,k,batch", [(4500, 4400, 16, None), (4200, 4608, 128, None), (4608, 4100, 144, None), (4100, 4300, 256, None),
                                         (1100, 1050, 400, 8), (384, 30000, 144, None), (100, 90, 272, 600), (300, 290, 256, 100)])
@pytest.mark.parametrize("a_tile,b_tile", [(False, True), (True, False), (False, False)])
def test_matmul_many_tiles(m, n, k, batch, a_tile, b_tile):
    """Many tiles of few blocks, whole and mostly empty ones, in batches."""
    announce(f"matmul_fp8 batch {batch} of {m} x {n} x {k} tiles {a_tile} {b_tile}")
    check_matmul(*operand(m, k, 1, a_tile, batch), *operand(n, k, 2, b_tile, batch), "bf16")


@pytest.mark.parametrize("shift", [1, 2, 4, 8, 15])
def test_matmul_alignment(shift):
    announce(f"matmul_fp8 at addresses {shift} bytes on")
    for m, n, k in ((9, 40, 256), (200, 300, 256)):
        (a, sa), (b, sb) = operand(m, k, 5, False), operand(n, k, 6, True)
        check_matmul(shifted(a.view(torch.uint8), shift).view(FP8), shifted(sa, shift % 4), b, sb, "bf16")
        check_matmul(a, sa, shifted(b.view(torch.uint8), shift).view(FP8), shifted(sb, shift % 4), "bf16")


@pytest.mark.parametrize("m,n,k", [(1, 64, 640), (24, 200, 1024), (256, 512, 2048), (300, 700, 1000), (1024, 1024, 128)])
def test_matmul_whole_numbers(m, n, k):
    """Whole numbers, scales of powers of two: every sum is exact."""
    import paper_2401_13660_amd as mb
    announce(f"matmul_fp8 in whole numbers {m} x {n} x {k}")
    g = torch.Generator().manual_seed(7)
    a = torch.randint(-8, 9, (m, k), generator=g).float()
    b = torch.randint(-8, 9, (n, k), generator=g).float()
    blocks = -(-k // 128)
    sa = 2.0 ** torch.randint(0, 4, (m, blocks), generator=g)
    sb = 2.0 ** torch.randint(0, 4, (-(-n // 128), blocks), generator=g)
    va = a * sa.repeat_interleave(128, 1)[:, :k]
    vb = b * sb.repeat_interleave(128, 1)[:, :k].repeat_interleave(128, 0)[:n]
    dev = lambda t: t.to("cuda:0")  # noqa: E731
    c = mb.matmul_fp8(dev(a).to(FP8), dev(sa.float()), dev(b).to(FP8), dev(sb.float()), out_dtype=torch.float32)
    assert torch.equal(c.cpu().double(), va.double() @ vb.double().t())


def test_matmul_special_values():
    """NaN and infinite scales reach their rows and columns and no others; nothing past k is taken in."""
    import paper_2401_13660_amd as mb
    announce("matmul_fp8: NaN, infinities, neighbours")
    for m, n, k in ((5, 70, 130), (200, 300, 272)):
        (a, sa), (b, sb) = operand(m, k, 8, False), operand(n, k, 9, False)
        clean = mb.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32)
        a.view(torch.uint8)[2, k - 1] = 0x7f
        b.view(torch.uint8)[n - 1, 0] = 0xff
        sb[10, 1] = float("inf")
        c = mb.matmul_fp8(a, sa, b, sb, out_dtype=torch.float32)
        torch.cuda.synchronize()
        hit = torch.zeros(m, n, dtype=torch.bool, device="cuda:0")
        hit[2], hit[:, n - 1] = True, True
        assert torch.isnan(c[hit]).all()
        hit[:, 10] = True
        assert not torch.isfinite(c[:, 10]).any() and torch.equal(c[~hit], clean[~hit])
        # rows of a larger buffer whose neighbours are NaN
        buf = torch.full((m + 2, k), 0x7f, dtype=torch.uint8, device="cuda:0")
        (a, sa), (b, sb) = operand(m, k, 8, False), operand(n, k, 9, False)
        buf[1:-1] = a.view(torch.uint8)
        assert torch.equal(mb.matmul_fp8(buf[1:-1].view(FP8), sa, b, sb, out_dtype=torch.float32), clean)


def test_matmul_out_and_edges():
    """A given output; what lies around it stays; k of 0; nothing."""
    import paper_2401_13660_amd as mb
    announce("matmul_fp8: outputs given, around them, empty sizes")
    for m, n, k in ((3, 37, 64), (150, 190, 128)):
        (a, sa), (b, sb) = operand(m, k, 1, False), operand(n, k, 2, True)
        for dtype in (torch.float32, torch.bfloat16):
            buf = torch.full((m * n + 64,), 7.0, device="cuda:0").to(dtype)
            out = buf[32:32 + m * n].view(m, n)
            assert mb.matmul_fp8(a, sa, b, sb, out=out) is out
            assert torch.equal(out, mb.matmul_fp8(a, sa, b, sb, out_dtype=dtype))
            assert (buf[:32] == 7).all() and (buf[32 + m * n:] == 7).all()
    z = mb.matmul_fp8(*operand(4, 0, 1, False), *operand(6, 0, 1, False))
    assert z.shape == (4, 6) and (z == 0).all()
    assert mb.matmul_fp8(*operand(0, 64, 1, False), *operand(6, 64, 1, False)).shape == (0, 6)


def test_matmul_large_output():
    """Columns past element 2^31 of the output, and rows past 2^31 bytes of an operand."""
    import paper_2401_13660_amd as mb
    announce("matmul_fp8 past 2^31 elements")
    m, n, k = 70000, 32768, 128
    (a, sa), (b, sb) = operand(m, k, 1, False), operand(n, k, 2, True)
    c = mb.matmul_fp8(a, sa, b, sb)
    part = mb.matmul_fp8(a[-130:].contiguous(), sa[-130:].contiguous(), b, sb)
    assert torch.equal(c[-130:], part)
    del c
    m, n, k = (1 << 20) + 100, 48, 2176
    a = torch.zeros(m, k, dtype=torch.uint8, device="cuda:0")
    sa = torch.ones(m, 17, device="cuda:0")
    x, xs = operand(100, k, 3, False)
    a[-100:], sa[-100:] = x.view(torch.uint8), xs
    b, sb = operand(n, k, 4, False)
    got = mb.matmul_fp8(a.view(FP8), sa, b, sb)[-100:]
    va, vb = values(x, xs), values(b, sb).transpose(1, 2).contiguous()
    ref, size = torch.matmul(va, vb)[0], torch.matmul(va.abs(), vb.abs())[0]
    assert ((got.double() - ref).abs() <= (256 + 20) * U * size + 7 * 2.0 ** -13 * eights(va, vb)[0] + 2.0 ** -8 * ref.abs()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,n", [((5, 40), 24), ((2, 70, 200), 130)])
def test_linear(shape, n, dtype):
    """The differentiable projection against the products of what quantising gives, and near the unrounded one."""
    import paper_2401_13660_amd as mb
    announce(f"linear_fp8 {shape} to {n} {dtype}")
    x = randn(shape, 1, dtype).requires_grad_()
    w = (randn((n, shape[-1]), 2, "f32") / shape[-1] ** 0.5).requires_grad_()
    dy = randn(shape[:-1] + (n,), 3, dtype)
    y = mb.linear_fp8(x, w)
    y.backward(dy)
    assert y.shape == shape[:-1] + (n,) and y.dtype == x.dtype and x.grad.dtype == x.dtype and w.grad.dtype == w.dtype

    def q(t, **kw):
        return values(*mb.quantize_fp8(t.detach().reshape(-1, t.shape[-1]), **kw))[0]
    tall = dict(transpose=True)
    want = {"y": (y, q(x) @ q(w, tile=True).t()),
            "dx": (x.grad, q(dy) @ q(w, tile=True, **tall).t()),
            "dw": (w.grad, q(dy, **tall) @ q(x, **tall).t())}
    plain = {"y": x.double().reshape(-1, shape[-1]) @ w.double().t(), "dx": dy.double().reshape(-1, n) @ w.double(),
             "dw": dy.double().reshape(-1, n).t() @ x.double().reshape(-1, shape[-1])}
    for k, (got, ref) in want.items():
        got = got.detach().double().view(ref.shape)
        tol = 1e-4 if got.dtype == torch.float32 else 2.0 ** -8
        assert (got - ref).norm() <= tol * ref.norm(), k
        # two factors, each within half a step (2^-4) of its own
        assert (got - plain[k]).norm() <= 2 * 2.0 ** -4 * 1.1 * plain[k].norm(), k
    g, = torch.autograd.grad(mb.linear_fp8(x, w).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice|once_differentiable"):
        g.square().sum().backward()


def test_matmul_of_millions():
    """A batch whose pieces of 64 rows would take a launch of 2^32 threads.  Whole numbers, exact."""
    import paper_2401_13660_amd as mb
    batch, m, k = (1 << 22) + 1, 65, 8
    announce(f"matmul_fp8 batch {batch} of ({m}, 1, {k})")
    a = torch.randint(-3, 4, (m, k), device="cuda:0").float()
    b = torch.randint(-3, 4, (batch, 1, k), device="cuda:0").float()
    one = torch.ones(batch, 1, 1, device="cuda:0")
    c = mb.matmul_fp8(a.to(FP8), one[0].expand(m, 1).contiguous(), b.to(FP8), one, out_dtype=torch.bfloat16)
    assert c.shape == (batch, m, 1) and torch.equal(c[:, :, 0].float(), b[:, 0] @ a.t())


def rows_of(shape):
    return int(np.prod(shape, dtype=np.int64))


@pytest.mark.parametrize("rows,k,n", [((0,), 7, 5), ((2, 0), 7, 5), ((3,), 0, 5), ((2, 3), 7, 0), ((0,), 0, 0), ((), 7, 5)])
def test_linear_of_nothing(rows, k, n):
    """Empty factors.  Values of 448 have a scale of 1: exact."""
    import paper_2401_13660_amd as mb
    announce(f"linear_fp8 {rows} x {k} to {n}")
    x, w = (torch.full(shape, 448.0, device="cuda:0", requires_grad=True) for shape in (rows + (k,), (n, k)))
    y = mb.linear_fp8(x, w)
    assert y.shape == rows + (n,) and (y == 448.0 ** 2 * k).all()
    y.backward(torch.full_like(y, 448.0))
    assert x.grad.shape == x.shape and (x.grad == 448.0 ** 2 * n).all()
    assert w.grad.shape == w.shape and (w.grad == 448.0 ** 2 * rows_of(rows)).all()

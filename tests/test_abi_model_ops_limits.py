"""What the entry points around the layers say of sizes at their limits, on the CPU: a workspace's size, or the refusal
that the call itself would give."""
import ctypes
import os

import pytest

import paper_2401_13660_amd as mb
from paper_2401_13660_amd import _binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmbscan.so not built")


no_gpu_only = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake addresses only on a machine without a GPU")
AT = [0x100000000000 * (i + 1) for i in range(12)]         # never used: the calls are refused


@no_gpu_only
@pytest.mark.parametrize("n,V,d", [(1 << 31, 256, 64), (1, 5, 1 << 32), (1 << 24, 256, 1 << 16), (3000, 200000, 1 << 30)])
def test_embedding_gradient_refused(n, V, d):
    lib = mb.load_library()
    assert lib.mb_embedding_bwd_workspace(n, V, d) == -2
    assert lib.mb_embedding_bwd(n, V, d, 1, 0, 0, 1.0, AT[0], AT[1], AT[2], None, None) == -2


@pytest.mark.parametrize("n,V,d", [((1 << 31) - 1, 256, 1), ((1 << 31) - 1, 70000, 63), (1 << 30, 256, 1), (1 << 30, 256, 64),
                                   (1 << 30, 256, 127), ((1 << 28) - 1, 300, 512), (127, 5, (1 << 30) - 1), (1, 5, (1 << 30) - 1)])
def test_embedding_gradient_taken(n, V, d):
    """What the header allows: fewer than 2^31 tokens, widths below 2^30, their product below 2^37."""
    assert n * d < 1 << 37
    assert mb.load_library().mb_embedding_bwd_workspace(n, V, d) > 0


def test_embedding_gradient_of_no_table():
    assert mb.load_library().mb_embedding_bwd_workspace(1 << 20, 0, 64) == 0


@no_gpu_only
@pytest.mark.parametrize("over", [dict(batch=2, dim=1 << 25), dict(batch=1 << 26, dim=1), dict(batch=0, dim=1 << 30),
                                  dict(batch=1 << 16, dim=1 << 10, seqlen=8192), dict(reserved=1), dict(reserved2=1), dict(width=5),
                                  dict(in_dtype=3)])
def test_convolution_gradient_refused(over):
    lib = mb.load_library()
    desc = B.ConvDesc(**dict(dict(batch=2, dim=8, seqlen=16, width=4, in_dtype=1, out_dtype=1, apply_silu=1, reserved=0,
                                  reserved2=0), **over))
    code = lib.mb_conv1d_bwd(ctypes.byref(desc), *AT[:4], *AT[4:6], *AT[6:10], None, None)
    assert code < 0 and lib.mb_conv1d_bwd_workspace(ctypes.byref(desc)) == code


@no_gpu_only
@pytest.mark.parametrize("b,n,V", [(1 << 20, 4, 2000), (1 << 22, 4, 256), (1 << 31, 0, 5), (1, 0, (1 << 31) - 1), (1 << 23, 0, 1025),
                                   (1 << 21, 0, 9000)])
def test_verification_refused(b, n, V):
    lib = mb.load_library()
    assert lib.mb_verify_sample_workspace(b, n, V) == -2
    assert lib.mb_verify_sample(b, n, V, 0, 1.0, AT[0], None, AT[1], None, AT[2], AT[3], AT[4], None, AT[5], None, None, None) == -2


@pytest.mark.parametrize("b,n,V", [((1 << 22) - 1, 4, 1024), (1 << 19, 4, 2000), ((1 << 22) - 1, 0, 4095), (1, 1 << 20, 8000)])
def test_verification_taken(b, n, V):
    size = mb.load_library().mb_verify_sample_workspace(b, n, V)
    assert size > 0 if V > 1024 else size == 0


@pytest.mark.parametrize("V,d", [(1, 1 << 34), (1, (1 << 34) - 1), (1, 1 << 45), (130000, 1 << 28)])
def test_no_tokens_and_wide_rows(V, d):
    """A workgroup per token and tile of columns (no workspace) counts a row's spans in 32 bits, so it takes no rows of this
    width: without tokens either, the table is set to zero by the launch that sorts them, which has a workspace."""
    assert mb.load_library().mb_embedding_bwd_workspace(0, V, d) > 0


def test_no_tokens_and_ordinary_rows():
    for V, d in ((1, 1), (256, 1792), (131072, 2304), (1, 1 << 19)):
        assert mb.load_library().mb_embedding_bwd_workspace(0, V, d) == 0

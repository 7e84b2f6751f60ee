"""The norm of rows without columns: a mean of nothing is NaN, in 1 / sqrt(mean + eps) too, and nothing else is written."""
import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("rows", [1, 5, 300])
def test_rstd(rows):
    import paper_2401_13660_amd as mb
    announce(f"rms_norm_fwd of {rows} rows without columns")
    rstd = torch.full((rows,), 7.0, device="cuda:0")
    assert mb.load_library().mb_rms_norm_fwd(rows, 0, 0, 0, 0, 1e-5, None, None, None, None, None, None, rstd.data_ptr(),
                                             torch.cuda.current_stream().cuda_stream) == 0
    assert torch.isnan(rstd).all()
    x = torch.empty(rows, 0, device="cuda:0")
    for res in (None, x):
        got = mb.rms_norm_fwd(x, torch.empty(0, device="cuda:0"), res, return_rstd=True)
        assert all(t.shape == (rows, 0) for t in got[:-1]) and got[-1].shape == (rows,) and torch.isnan(got[-1]).all()
    q, s = mb.rms_norm_fp8(x)
    assert q.shape == s.shape == (rows, 0)
    a, w = x.clone().requires_grad_(), torch.empty(0, device="cuda:0", requires_grad=True)
    mb.rms_norm(a, w).sum().backward()
    assert a.grad.shape == (rows, 0) and w.grad.shape == (0,)

"""The gradient's C entry point asked for a residual's gradient where h has none of its own (dh NULL): what zeros for it give."""
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_embedding import DT
from test_gpu_rms_norm import grad_inputs

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
CODE = {"f32": 0, "bf16": 1}


@pytest.mark.parametrize("rows,dim", [(1, 1), (7, 300), (300, 1792), (9, 1003), (5, 5000), (3, 16384), (4, 20001)])
@pytest.mark.parametrize("dy,h,dx", [("bf16", "f32", "bf16"), ("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32")])
@pytest.mark.parametrize("weighted", [True, False])
def test_residual_without_dh(rows, dim, dy, h, dx, weighted):
    import paper_2401_13660_amd as mb
    announce(f"mb_rms_norm_bwd ({rows}, {dim}) dy {dy} h {h} dx {dx}, dresidual without dh")
    lib = mb.load_library()
    g = grad_inputs(rows, dim, dy, h, 1)
    ws = torch.empty(max(16, lib.mb_rms_norm_bwd_workspace(rows, dim)), dtype=torch.uint8, device="cuda:0")
    got = []
    for dh in (None, torch.zeros_like(g["h"])):
        out = dict(dx=torch.full_like(g["h"], 7.0, dtype=DT[dx]), dres=torch.full_like(g["h"], 7.0), dw=torch.full((dim,), 7.0, device="cuda:0"))
        st = lib.mb_rms_norm_bwd(rows, dim, CODE[dy], CODE[h], CODE[dx], g["dy"].data_ptr(), g["h"].data_ptr(), g["rstd"].data_ptr(),
                                 g["w"].data_ptr() if weighted else None, None if dh is None else dh.data_ptr(), out["dx"].data_ptr(),
                                 out["dres"].data_ptr(), out["dw"].data_ptr(), ws.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0
        got.append(out)
    for k in got[0]:
        assert torch.equal(got[0][k], got[1][k]), k
    if h == dx:
        assert torch.equal(got[0]["dx"], got[0]["dres"])
    ref = mb.rms_norm_bwd(g["dy"], g["h"], g["rstd"], g["w"] if weighted else None, dx_dtype=DT[dx])
    assert torch.equal(got[0]["dx"], ref["dx"])

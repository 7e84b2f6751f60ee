"""The C ABI of the operators around the layers with the workspace left to the call (NULL), and with the least one given:
the same bits as through the binding, and nothing written past it."""
import ctypes

import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_clip import tensors
from test_gpu_conv_bwd import inputs
from test_gpu_embedding import randn
from test_gpu_verify_sample import case

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
GUARD = 4096


def ptr(t):
    return None if t is None else t.data_ptr()


class Space:
    """A workspace of exactly `size` bytes between guards, or none."""

    def __init__(self, size, given):
        assert size >= 0
        self.size, self.given = size, given
        self.buf = torch.full((size + 2 * GUARD,), 0x5A, dtype=torch.uint8, device="cuda:0")
        self.at = self.buf.data_ptr() + GUARD if given else None

    def check(self):
        torch.cuda.synchronize()
        assert (self.buf[:GUARD] == 0x5A).all() and (self.buf[GUARD + self.size:] == 0x5A).all()


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("n,V,d", [(0, 9, 4), (700, 256, 40), (5000, 300, 17), (40000, 70000, 3)])
def test_embedding_bwd(given, n, V, d):
    import paper_2401_13660_amd as mb
    announce(f"mb_embedding_bwd n={n} V={V} workspace given: {given}")
    lib = mb.load_library()
    t = torch.randint(0, V, (n,), device="cuda:0", dtype=torch.int32)
    dy, out = randn((n, d), 1, "bf16"), torch.empty(V, d, device="cuda:0")
    ws = Space(lib.mb_embedding_bwd_workspace(n, V, d), given)
    assert lib.mb_embedding_bwd(n, V, d, 1, 1, 0, 0.5, ptr(t), ptr(dy), ptr(out), ws.at, stream()) == 0
    ws.check()
    assert torch.equal(out, mb.embedding_bwd(t, dy, V, scale=0.5))


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("shape", [(2, 5, 9), (1, 7, 600), (3, 4, 5001)])
def test_conv1d_bwd(given, shape):
    import paper_2401_13660_amd as mb
    from paper_2401_13660_amd._binding import ConvDesc
    announce(f"mb_conv1d_bwd {shape} workspace given: {given}")
    lib = mb.load_library()
    a = inputs(*shape, 4, "bf16", "f32", 2)
    ref = mb.conv1d_bwd(a["x"], a["w"], a["dy"], a["bias"], a["state"], a["dstate_out"])
    out = {k: torch.empty_like(v) for k, v in ref.items()}
    desc = ConvDesc(*shape, 4, 1, 0, 1, 0, 0)
    ws = Space(lib.mb_conv1d_bwd_workspace(ctypes.byref(desc)), given)
    assert lib.mb_conv1d_bwd(ctypes.byref(desc), ptr(a["x"]), ptr(a["w"]), ptr(a["bias"]), ptr(a["state"]), ptr(a["dy"]),
                             ptr(a["dstate_out"]), ptr(out["dx"]), ptr(out["dw"]), ptr(out["dbias"]), ptr(out["dstate"]),
                             ws.at, stream()) == 0
    ws.check()
    for k in ref:
        assert torch.equal(out[k], ref[k]), k


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("count", [0, 1, 64, 65, 300])
def test_norm_and_clip(given, count):
    import paper_2401_13660_amd as mb
    announce(f"mb_grad_norm and mb_clip_grad_norm of {count} tensors, workspace given: {given}")
    lib = mb.load_library()
    g = tensors([(i * 131) % 9000 for i in range(count)], ["bf16", "f32"] * ((count + 1) // 2), 3)
    ptrs = (ctypes.c_void_p * max(count, 1))(*[t.data_ptr() for t in g])
    sizes = (ctypes.c_int64 * max(count, 1))(*[t.numel() for t in g])
    types = (ctypes.c_int32 * max(count, 1))(*[1 if t.dtype == torch.bfloat16 else 0 for t in g])
    ref = mb.grad_norm(g) if count else torch.zeros((), device="cuda:0")
    clipped = [t.clone() for t in g]
    if count:
        mb.clip_grad_norm(clipped, 0.25)
    norm = torch.full((2,), -1.0, device="cuda:0")
    ws = Space(lib.mb_grad_norm_workspace(count), given)
    assert lib.mb_grad_norm(count, ptrs, sizes, types, norm.data_ptr(), ws.at, stream()) == 0
    assert lib.mb_clip_grad_norm(count, ptrs, None, sizes, types, 0.25, 1e-6, norm.data_ptr() + 4, ws.at, stream()) == 0
    ws.check()
    assert norm[0] == ref and norm[1] == ref
    for x, y in zip(g, clipped):
        assert torch.equal(x, y)


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("B,n,V", [(3, 4, 256), (3, 4, 1025), (2, 0, 40000)])
def test_verify_sample(given, B, n, V):
    import paper_2401_13660_amd as mb
    announce(f"mb_verify_sample ({B}, {n}, {V}) workspace given: {given}")
    lib = mb.load_library()
    a = case(B, n, V, "bf16", seed=4)
    ref = mb.verify_sample(a["logits"], a["draft"], a["uniform"], a["noise"], a["draft_logits"], temperature=0.8)
    acc, nxt = (torch.full((B,), -7, dtype=torch.int32, device="cuda:0") for _ in range(2))
    ws = Space(lib.mb_verify_sample_workspace(B, n, V), given)
    # neither last_pos nor probabilities asked for
    assert lib.mb_verify_sample(B, n, V, 1, 0.8, ptr(a["logits"]), ptr(a["draft_logits"]), ptr(a["draft"]), None,
                                ptr(a["uniform"]), ptr(a["noise"]), ptr(acc), None, ptr(nxt), None, ws.at, stream()) == 0
    ws.check()
    assert torch.equal(acc, ref[0]) and torch.equal(nxt, ref[2])

"""The operators around the layers on other streams than the default one, and in HIP graphs: each call works on the
current stream, and a replay gives the eager call's bits, with eager work between the replays."""
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_clip import tensors
from test_gpu_conv_bwd import inputs
from test_gpu_embedding import randn
from test_gpu_verify_sample import case

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def calls(seed):
    """name: (a call that returns tensors)"""
    import paper_2401_13660_amd as mb
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    tokens = torch.randint(0, 256, (3000,), generator=g, device="cuda:0").to(torch.uint8)
    wide = torch.randint(0, 5000, (3000,), generator=g, device="cuda:0").int()
    W, dy = randn((256, 200), seed, "bf16"), randn((3000, 200), seed + 1, "bf16")
    conv = inputs(2, 40, 1500, 4, "bf16", "bf16", seed)
    grads = tensors([70000, 33, 5000] * 60, ["f32", "bf16", "f32"] * 60, seed)
    outs = [torch.empty_like(t) for t in grads]
    small, large = case(9, 5, 256, seed=seed), case(3, 4, 9000, "bf16", seed=seed)

    def conv_call():
        r = mb.conv1d_bwd(conv["x"], conv["w"], conv["dy"], conv["bias"], conv["state"], conv["dstate_out"])
        return [r[k] for k in sorted(r)]

    def verify(a):
        return list(mb.verify_sample(a["logits"], a["draft"], a["uniform"], a["noise"], a["draft_logits"], return_probs=True))
    return {
        "embedding_fwd": lambda: [mb.embedding_fwd(tokens, W, scale=2.0)],
        "embedding_bwd": lambda: [mb.embedding_bwd(tokens, dy, 256)],
        "embedding_bwd_wide": lambda: [mb.embedding_bwd(wide, dy, 5000)],
        "conv1d_bwd": conv_call,
        "grad_norm": lambda: [mb.grad_norm(grads)],
        "clip_grad_norm": lambda: [mb.clip_grad_norm(grads, 1.0, out=outs)] + outs[:3],
        "verify_sample": lambda: verify(small),
        "verify_sample_wide": lambda: verify(large),
    }


NAMES = ["embedding_fwd", "embedding_bwd", "embedding_bwd_wide", "conv1d_bwd", "grad_norm", "clip_grad_norm", "verify_sample",
         "verify_sample_wide"]


def test_two_streams():
    announce("operators around the layers on two streams at once")
    sets = [calls(1), calls(2)]
    serial = [{k: [t.clone() for t in s[k]()] for k in NAMES} for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for s, c in zip(streams, sets):
        with torch.cuda.stream(s):
            got.append({k: c[k]() for k in NAMES})
    torch.cuda.synchronize()
    for a, b in zip(got, serial):
        for k in NAMES:
            for x, y in zip(a[k], b[k]):
                assert torch.equal(x, y), k


@pytest.mark.parametrize("name", NAMES)
def test_graph(name):
    announce(f"HIP graph of {name}")
    call = calls(3)[name]
    ref = [t.clone() for t in call()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph, held = torch.cuda.CUDAGraph(), {}
    with torch.cuda.graph(graph):
        held["out"] = call()
    for r in range(4):
        call()                                              # eager work between replays
        for t in held["out"]:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(held["out"], ref):
            assert torch.equal(x, y), f"replay {r}"

"""The example that trains and samples a small byte model with the library's operators together."""
import importlib.util
import os

import pytest
import torch

from gpu_util import announce, has_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "byte_model.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("byte_model", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_learns_and_samples(example):
    """The loss falls, and after speculative rounds in which the sequences keep different numbers of drafted bytes the
    carried states are those of the bytes that were kept."""
    announce("examples/byte_model.py: training and speculative sampling")
    torch.manual_seed(0)
    text = torch.frombuffer(bytearray(open(PATH, "rb").read()), dtype=torch.uint8).to("cuda:0")
    model = example.ByteModel(width=32)
    losses, norms = example.train(model, text, 60)
    assert losses[0] > 4.0 and sum(losses[-10:]) / 10 < 0.75 * losses[0]
    assert all(0 < n < 1e3 for n in norms)
    prompt = torch.stack([text[i * 40:i * 40 + 17] for i in range(5)])
    out, states, accepted = example.generate(model, example.pair_logits(text), prompt, rounds=6)
    assert len(set(accepted.flatten().tolist())) > 2 and accepted.min() >= 0 and accepted.max() <= 8
    for b, row in enumerate(out):
        assert len(row) == 17 + 6 + int(accepted[:, b].sum()) and all(0 <= t < 256 for t in row)
        tokens = torch.tensor([row[:-1]], dtype=torch.int32, device="cuda:0")
        _, seen = model.extend(tokens, model.empty(1))
        last = torch.tensor([len(row) - 2], dtype=torch.int32, device="cuda:0")
        for layer, (conv, scan) in enumerate(example.Block.at(s, last) for s in seen):
            assert torch.allclose(conv[0], states[layer][0][b], rtol=1e-3, atol=1e-3)
            assert torch.allclose(scan[0], states[layer][1][b], rtol=1e-3, atol=1e-3)


def test_gradients_reach_every_parameter(example):
    announce("examples/byte_model.py: gradients")
    torch.manual_seed(1)
    model = example.ByteModel(width=16, layers=1)
    tokens = torch.randint(0, 256, (2, 32), device="cuda:0")
    model(tokens).square().mean().backward()
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all() and p.grad.abs().max() > 0, name

"""A small byte-level model of Mamba blocks, trained and then sampled by speculation, with the library's operators
running together: the embedding, the convolution and the scan with their gradients, the clipping of all gradients; then
drafts from byte-pair counts, the convolution and the scan over a draft from their carried states, the verification
against the model's probabilities, and the states at the last accepted byte.

    python examples/byte_model.py [steps]
"""
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2401_13660_amd as mb  # noqa: E402

VOCAB, N, K = 256, 16, 4        # byte values, states per channel, taps of the convolution
DEV = "cuda:0"


class Block(torch.nn.Module):
    """in_proj, causal convolution and Swish, x_proj and dt_proj, scan with skip and gate, out_proj, residual."""

    def __init__(self, width):
        super().__init__()
        D, r = 2 * width, max(1, width // 16)
        self.r = r

        def weight(*shape):
            return torch.nn.Parameter(torch.randn(*shape, device=DEV) / math.sqrt(shape[1]))
        self.norm = torch.nn.Parameter(torch.ones(width, device=DEV))
        self.in_proj, self.x_proj = weight(2 * D, width), weight(r + 2 * N, D)
        self.dt_proj, self.out_proj = weight(D, r), weight(width, D)
        self.taps = torch.nn.Parameter((torch.rand(D, K, device=DEV) - 0.5) * 2 / math.sqrt(K))
        self.bias = torch.nn.Parameter(torch.zeros(D, device=DEV))
        self.A_log = torch.nn.Parameter(torch.arange(1, N + 1, device=DEV).float().log().repeat(D, 1))
        self.D = torch.nn.Parameter(torch.ones(D, device=DEV))
        dt = torch.exp(torch.rand(D, device=DEV) * math.log(100) + math.log(1e-3))
        self.dt_bias = torch.nn.Parameter(torch.log(torch.expm1(dt)))

    def split(self, h):
        """(batch, L, width) -> the convolution's input and the gate, (batch, D, L)."""
        h = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * self.norm
        x, z = (h @ self.in_proj.t()).transpose(1, 2).chunk(2, 1)
        return x.contiguous(), z.contiguous()

    def select(self, u):
        """The scan's timestep, input and output projections of u (batch, D, L)."""
        dbc = u.transpose(1, 2) @ self.x_proj.t()
        delta = (dbc[..., :self.r] @ self.dt_proj.t()).transpose(1, 2).contiguous()
        B, C = dbc[..., self.r:].transpose(1, 2).chunk(2, 1)
        return delta, -torch.exp(self.A_log), B.contiguous(), C.contiguous()

    def forward(self, h):
        x, z = self.split(h)
        u, _ = mb.causal_conv1d(x, self.taps, self.bias)
        delta, A, B, C = self.select(u)
        y, _ = mb.selective_scan(u, delta, A, B, C, self.D, self.dt_bias, z)
        return h + y.transpose(1, 2) @ self.out_proj.t()

    def extend(self, h, state):
        """The block over new bytes from a carried (convolution, scan) state.  Returns the outputs and what `at` needs
        to find the state after any of the bytes."""
        conv, scan = state
        x, z = self.split(h)
        u = mb.conv1d(x, self.taps, self.bias, conv)
        delta, A, B, C = self.select(u)
        args = (u, delta, A, B, C, self.D, self.dt_bias, z, scan)
        return h + mb.scan_fwd(*args).transpose(1, 2) @ self.out_proj.t(), (torch.cat([conv, x], 2), args)

    @staticmethod
    def at(seen, last):
        """The state after byte last[b] of each sequence."""
        ext, args = seen
        where = last[:, None, None] + 1 + torch.arange(K - 1, device=DEV)       # the K - 1 inputs up to that byte
        conv = ext.gather(2, where.expand(-1, ext.shape[1], -1).long()).contiguous()
        return conv, mb.scan_fwd(*args, positions=last[None].int())[1][0]


class ByteModel(torch.nn.Module):
    def __init__(self, width=64, layers=2):
        super().__init__()
        self.width = width
        self.table = torch.nn.Parameter(torch.randn(VOCAB, width, device=DEV) / math.sqrt(width))
        self.blocks = torch.nn.ModuleList(Block(width) for _ in range(layers))

    def embed(self, tokens):
        return mb.embedding(tokens, self.table, scale=math.sqrt(self.width))

    def forward(self, tokens):
        h = self.embed(tokens)
        for block in self.blocks:
            h = block(h)
        return h @ self.table.t()

    def empty(self, batch):
        D = 2 * self.width
        return [(torch.zeros(batch, D, K - 1, device=DEV), torch.zeros(batch, D, N, device=DEV)) for _ in self.blocks]

    @torch.no_grad()
    def extend(self, tokens, states):
        h, seen = mb.embedding_fwd(tokens, self.table, scale=math.sqrt(self.width)), []
        for block, state in zip(self.blocks, states):
            h, s = block.extend(h, state)
            seen.append(s)
        return h @ self.table.t(), seen


def train(model, text, steps, batch=8, length=256, max_norm=1.0):
    """Steps on windows of the text.  Returns the losses and the gradients' norms."""
    params = list(model.parameters())
    opt = torch.optim.AdamW(params, lr=3e-3, betas=(0.9, 0.95))
    g = torch.Generator().manual_seed(0)
    losses, norms = [], []
    for _ in range(steps):
        starts = torch.randint(0, len(text) - length - 1, (batch,), generator=g)
        window = torch.stack([text[s:s + length + 1] for s in starts.tolist()])
        logits = model(window[:, :-1].contiguous())
        loss = F.cross_entropy(logits.reshape(-1, VOCAB), window[:, 1:].reshape(-1).long())
        opt.zero_grad()
        loss.backward()
        norms.append(mb.clip_grad_norm([p.grad for p in params], max_norm))
        opt.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist(), torch.stack(norms).tolist()


def pair_logits(text):
    """A drafter: the logarithms of byte-pair frequencies, every pair counted at least a little."""
    counts = torch.full((VOCAB, VOCAB), 0.05, device=DEV)
    t = text.long()
    counts.view(-1).index_add_(0, t[:-1] * VOCAB + t[1:], torch.ones(len(t) - 1, device=DEV))
    return (counts / counts.sum(1, keepdim=True)).log()


@torch.no_grad()
def generate(model, drafter, prompt, rounds, drafts=8, temperature=1.0, seed=0):
    """Speculative sampling of a batch of prompts (batch, L) of bytes.  Returns each sequence's bytes, the states after
    all of them but the last, and the drafted bytes accepted per round."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    b = prompt.shape[0]
    logits, seen = model.extend(prompt[:, :-1].contiguous(), model.empty(b))
    last = torch.full((b,), prompt.shape[1] - 2, dtype=torch.int32, device=DEV)
    states = [Block.at(s, last) for s in seen]
    cur, out, accepted_all = prompt[:, -1].int(), [row.tolist() for row in prompt], []
    for _ in range(rounds):
        chunk, draft_logits = [cur], []
        for _ in range(drafts):                             # the drafter samples from the same temperature
            lg = drafter[chunk[-1].long()]
            draft_logits.append(lg)
            noise = torch.empty(b, VOCAB, device=DEV).exponential_(generator=g)
            chunk.append((lg / temperature - noise.log()).argmax(1).int())
        chunk = torch.stack(chunk, 1)
        logits, seen = model.extend(chunk, states)
        accepted, _, following = mb.verify_sample(
            logits, chunk[:, 1:].contiguous(), torch.rand(b, drafts, generator=g, device=DEV),
            torch.empty(b, VOCAB, device=DEV).exponential_(generator=g), torch.stack(draft_logits, 1),
            temperature=temperature)
        states = [Block.at(s, accepted) for s in seen]      # byte 0 of the chunk is the one before the drafts
        cur = following
        accepted_all.append(accepted)
        for row, c, n, f in zip(out, chunk.tolist(), accepted.tolist(), following.tolist()):
            row += c[1:1 + n] + [f]
    return out, states, torch.stack(accepted_all)


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 300
    torch.manual_seed(0)
    data = open(os.path.abspath(__file__), "rb").read()
    text = torch.frombuffer(bytearray(data), dtype=torch.uint8).to(DEV)
    model = ByteModel()
    losses, norms = train(model, text, steps)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f} nats per byte over {steps} steps; gradient norm {norms[-1]:.2f}")
    prompt = text[1000:1256].repeat(4, 1)
    out, _, accepted = generate(model, pair_logits(text), prompt, rounds=24)
    print(f"{accepted.float().mean():.2f} of 8 drafted bytes accepted per round")
    print(bytes(out[0][200:]).decode("utf-8", "replace"))


if __name__ == "__main__":
    main()

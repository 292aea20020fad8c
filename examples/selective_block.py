"""A small language model of selective-scan blocks, trained and served with the library's calls:

    python examples/selective_block.py

A block is a norm, a projection to an input and a gate, the short convolution over the input, the projections of what the scan takes from it, the scan, and the projection
back.  Training runs the differentiable forms and clips the gradients together; serving reads prompts of different lengths packed behind one another, keeps the last inputs of the
convolution and the scan's states for each sequence, and goes on token by token.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1811_09736_amd import autograd, binding  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, width, inner, states, taps, rank, dtype):
        super().__init__()

        def matrix(*shape):
            return torch.nn.Parameter((torch.randn(*shape, device="cuda") * shape[-1] ** -0.5).to(dtype))

        self.states, self.rank = states, rank
        self.norm = torch.nn.Parameter(torch.ones(width, device="cuda", dtype=dtype))
        self.into = matrix(2 * inner, width)
        self.taps = matrix(inner, taps)
        self.taps_bias = torch.nn.Parameter(torch.zeros(inner, device="cuda", dtype=dtype))
        self.select = matrix(rank + 2 * states, inner)
        self.step = matrix(inner, rank)
        # steps between a thousandth and a tenth, rates from 1 to the number of states (learned by their logarithm, so that they stay negative)
        target = torch.exp(torch.rand(inner, device="cuda") * math.log(100.0) + math.log(1e-3))
        self.step_bias = torch.nn.Parameter(target + torch.log(-torch.expm1(-target)))
        self.log_rate = torch.nn.Parameter(torch.log(torch.arange(1, states + 1, device="cuda", dtype=torch.float32)).repeat(inner, 1))
        self.skip = torch.nn.Parameter(torch.ones(inner, device="cuda"))
        self.back = matrix(width, inner)

    def inputs(self, h):
        """What the scan takes beside h: dt, b and c (of one group)."""
        dt, b, c = (h @ self.select.T).split((self.rank, self.states, self.states), -1)
        return dt @ self.step.T, b.unsqueeze(-2), c.unsqueeze(-2)

    def forward(self, y):
        x, gate = (y @ self.into.T).chunk(2, -1)
        h, _ = autograd.causal_conv(x, self.taps, self.taps_bias)
        dt, b, c = self.inputs(h)
        out, _ = autograd.selective_scan(h, dt, -self.log_rate.exp(), b, c, skip=self.skip, gate=gate, dt_bias=self.step_bias)
        return out @ self.back.T

    def serve(self, y, state, offsets=None):
        """Packed prompts (offsets given) or one further token for every sequence; state: [last inputs, states], which go on."""
        x, gate = (y @ self.into.T).chunk(2, -1)
        if offsets is not None:
            h, state[0] = binding.causal_conv(x, self.taps, self.taps_bias, offsets=offsets, state=state[0], final_state=True)
        else:
            h = binding.causal_conv_step(x, self.taps, state[0], self.taps_bias)
        dt, b, c = self.inputs(h)
        args = (h, dt, -self.log_rate.exp(), b, c)
        given = {"skip": self.skip, "gate": gate, "dt_bias": self.step_bias}
        if offsets is not None:
            out, state[1] = binding.selective_scan(*args, **given, offsets=offsets, state=state[1], final_state=True)
        else:
            out = binding.selective_scan_step(*args, state[1], **given)
        return out @ self.back.T


class Model(torch.nn.Module):
    def __init__(self, vocabulary=64, width=64, inner=128, states=16, taps=4, rank=8, blocks=2, dtype=torch.bfloat16):
        super().__init__()
        self.embedding = torch.nn.Parameter(torch.randn(vocabulary, width, device="cuda").to(dtype))
        self.blocks = torch.nn.ModuleList(Block(width, inner, states, taps, rank, dtype) for _ in range(blocks))
        self.norm = torch.nn.Parameter(torch.ones(width, device="cuda", dtype=dtype))
        self.head = torch.nn.Parameter((torch.randn(vocabulary, width, device="cuda") * width ** -0.5).to(dtype))

    def forward(self, tokens):
        """Logits of [batch, length] tokens, with gradients."""
        total, y = self.embedding[tokens], None
        for block in self.blocks:
            if y is None:
                h = autograd.rms_norm(total, block.norm)
            else:
                h, total = autograd.rms_norm(y, block.norm, total)
            y = block(h)
        return autograd.rms_norm(y, self.norm, total)[0] @ self.head.T

    @torch.no_grad()
    def serve(self, tokens, states, offsets=None):
        """Logits of packed prompts (offsets given), or of one further token for every sequence; the states go on."""
        total, y = self.embedding[tokens], None
        for block, state in zip(self.blocks, states):
            if y is None:
                h = binding.rms_norm(total, block.norm)
            else:
                h, total = binding.rms_norm(y, block.norm, residual=total)
            y = block.serve(h, state, offsets)
        return binding.rms_norm(y, self.norm, residual=total)[0] @ self.head.T

    def states(self, sequences):
        return [[torch.zeros(sequences, b.taps.shape[1] - 1, b.taps.shape[0], device="cuda", dtype=b.taps.dtype),
                 torch.zeros(sequences, *b.log_rate.shape, device="cuda")] for b in self.blocks]


def sequences(count, length, vocabulary, gen):
    """Counting on in steps of 3 from a random start; each token in eight is replaced by a random one."""
    start = torch.randint(0, vocabulary, (count, 1), generator=gen, device="cuda")
    tokens = (start + 3 * torch.arange(length, device="cuda")) % vocabulary
    noise = torch.rand(count, length, generator=gen, device="cuda") < 0.125
    return torch.where(noise, torch.randint(0, vocabulary, (count, length), generator=gen, device="cuda"), tokens)


def train(model, steps, batch=16, length=96, limit=1.0, seed=0):
    """The losses of `steps` steps of Adam, and the gradients' norms in front of the clipping."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses, norms = [], []
    for _ in range(steps):
        tokens = sequences(batch, length + 1, model.head.shape[0], gen)
        loss = torch.nn.functional.cross_entropy(model(tokens[:, :-1]).float().flatten(0, 1), tokens[:, 1:].flatten())
        optimizer.zero_grad()
        loss.backward()
        norms.append(binding.clip_gradients([p.grad for p in model.parameters()], limit).item())
        optimizer.step()
        losses.append(loss.item())
    return losses, norms


def generate(model, prompts, count):
    """The most likely `count` further tokens of each prompt (a list of lists)."""
    offsets = torch.tensor([0] + [len(p) for p in prompts], device="cuda").cumsum(0)
    states = model.states(len(prompts))
    logits = model.serve(torch.tensor([t for p in prompts for t in p], device="cuda"), states, offsets)
    token = logits[offsets[1:] - 1].argmax(-1)
    got = [token]
    for _ in range(count - 1):
        token = model.serve(token, states).argmax(-1)
        got.append(token)
    return torch.stack(got, 1).tolist()


if __name__ == "__main__":
    torch.manual_seed(0)
    model = Model()
    losses, norms = train(model, 200)
    print("loss: first step %.3f, last %.3f; gradient norm %.2f, %.2f" % (losses[0], losses[-1], norms[0], norms[-1]))
    prompts = [list(range(5, 40, 3)), list(range(20, 60, 3))]
    for prompt, more in zip(prompts, generate(model, prompts, 8)):
        print("prompt", prompt, "goes on with", more)

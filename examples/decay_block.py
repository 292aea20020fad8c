"""A small language model of linear-attention blocks, trained and served with the library's calls:

    python examples/decay_block.py

Training runs the differentiable forms (the norm with the residual's addition, attention, their gradients).  Serving reads prompts of different lengths packed
behind one another, keeps one state a sequence, whatever its length, and goes on token by token; the norms in front of the products give e4m3
codes with a scale for each row, which here are multiplied out again (a product in 8 bits would take them as they are).
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1811_09736_amd import autograd, binding  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, vocabulary=64, width=128, heads=2, blocks=2, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.dim = heads, width // heads
        parameter = lambda *shape: torch.nn.Parameter(torch.randn(*shape, device="cuda", dtype=torch.float32).mul_(shape[-1] ** -0.5).to(dtype))  # noqa: E731
        self.embedding = torch.nn.Parameter(torch.randn(vocabulary, width, device="cuda").to(dtype))
        self.norms = torch.nn.ParameterList(torch.nn.Parameter(torch.ones(width, device="cuda", dtype=dtype)) for _ in range(blocks + 1))
        self.qkv = torch.nn.ParameterList(parameter(3 * width, width) for _ in range(blocks))
        self.out = torch.nn.ParameterList(parameter(width, width) for _ in range(blocks))
        self.head = parameter(vocabulary, width)
        # heads that look back over 4 tokens to heads that look back over 64
        self.register_buffer("log_decay", torch.log1p(-torch.exp2(-torch.linspace(2.0, 6.0, heads, device="cuda"))))

    def split(self, y, weight):
        return (y @ weight.T).unflatten(-1, (3, self.heads, self.dim)).unbind(-3)

    def forward(self, tokens):
        """Logits of [batch, length] tokens, with gradients."""
        total, y = self.embedding[tokens], None
        for norm, qkv, out in zip(self.norms, self.qkv, self.out):
            if y is None:
                h = autograd.rms_norm(total, norm)
            else:
                h, total = autograd.rms_norm(y, norm, total)
            q, k, v = self.split(h, qkv)
            y = autograd.linear_attention(q, k, v, self.log_decay)[0].flatten(-2) @ out.T
        return autograd.rms_norm(y, self.norms[-1], total)[0] @ self.head.T

    @torch.no_grad()
    def serve(self, tokens, states, offsets=None):
        """Logits of packed prompts (offsets given), or of one further token for every sequence; the states go on."""
        total, y = self.embedding[tokens], None
        for i, (norm, qkv, out) in enumerate(zip(self.norms, self.qkv, self.out)):
            codes, scales, *sums = binding.rms_norm_quantized(total if y is None else y, norm, residual=None if y is None else total)
            total = sums[0] if sums else total
            q, k, v = self.split((codes.float() * scales).to(total.dtype), qkv)
            if offsets is None:
                o = binding.linear_attention_step(q, k, v, self.log_decay, states[i])
            else:
                o, states[i] = binding.linear_attention(q, k, v, self.log_decay, offsets=offsets, state=states[i], final_state=True)
            y = o.flatten(-2) @ out.T
        return binding.rms_norm(y, self.norms[-1], residual=total)[0] @ self.head.T

    def states(self, sequences):
        return [torch.zeros(sequences, self.heads, self.dim, self.dim, device="cuda") for _ in self.qkv]


def sequences(count, length, vocabulary, gen):
    """Counting on in steps of 3 from a random start; each token in eight is replaced by a random one."""
    start = torch.randint(0, vocabulary, (count, 1), generator=gen, device="cuda")
    tokens = (start + 3 * torch.arange(length, device="cuda")) % vocabulary
    noise = torch.rand(count, length, generator=gen, device="cuda") < 0.125
    return torch.where(noise, torch.randint(0, vocabulary, (count, length), generator=gen, device="cuda"), tokens)


def train(model, steps, batch=16, length=96, seed=0):
    """The losses of `steps` steps of Adam."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for _ in range(steps):
        tokens = sequences(batch, length + 1, model.head.shape[0], gen)
        loss = torch.nn.functional.cross_entropy(model(tokens[:, :-1]).float().flatten(0, 1), tokens[:, 1:].flatten())
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
    return losses


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
    losses = train(model, 200)
    print("loss: first step %.3f, last %.3f" % (losses[0], losses[-1]))
    prompts = [list(range(5, 40, 3)), list(range(20, 60, 3))]
    for prompt, more in zip(prompts, generate(model, prompts, 8)):
        print("prompt", prompt, "goes on with", more)

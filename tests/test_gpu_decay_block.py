"""The example of examples/decay_block.py: gradients against plain torch in 64 bits, training, and serving that gives what the model gives."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("decay_block", os.path.join(ROOT, "examples", "decay_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(model, tokens, parameters):
    """The model's logits in 64 bits by elementary operations."""
    total, y = parameters["embedding"][tokens], None

    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w

    t = torch.arange(tokens.shape[1], device="cuda", dtype=torch.float64)
    rel = t[:, None] - t[None, :]
    weights = torch.where(rel >= 0, torch.exp(model.log_decay.double()[:, None, None] * rel.clamp(min=0)), 0.0)
    for i in range(len(model.qkv)):
        total = total if y is None else total + y
        q, k, v = (norm(total, parameters[f"norms.{i}"]) @ parameters[f"qkv.{i}"].T).unflatten(-1, (3, model.heads, model.dim)).unbind(-3)
        q, k, v = q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2)
        o = torch.matmul(torch.matmul(q, k.transpose(2, 3)) * weights, v) * model.dim ** -0.5
        y = o.transpose(1, 2).flatten(-2) @ parameters[f"out.{i}"].T
    return norm(total + y, parameters[f"norms.{len(model.qkv)}"]) @ parameters["head"].T


def test_gradients_of_the_whole_model(block):
    torch.manual_seed(1)
    model = block.Model(vocabulary=32, width=64, heads=2, blocks=2)
    tokens = torch.randint(0, 32, (3, 70), device="cuda")
    target = torch.randn(3, 70, 32, device="cuda")
    logits = model(tokens)
    (logits.float() * target).sum().backward()
    parameters = {n: p.detach().double().requires_grad_() for n, p in model.named_parameters()}
    want = plain(model, tokens, parameters)
    (want * target.double()).sum().backward()
    # every activation on the way is rounded to bfloat16, 2^-9 relative on average: two blocks of a handful of roundings each
    assert (logits.double() - want).norm() <= 0.03 * want.norm()
    for n, p in model.named_parameters():
        assert p.grad is not None and (p.grad.double() - parameters[n].grad).norm() <= 0.05 * parameters[n].grad.norm(), n


def test_training_learns(block):
    torch.manual_seed(0)
    losses = block.train(block.Model(), 120)
    assert losses[-1] < 0.6 * losses[0]


def test_serving_goes_on_like_the_prompt(block):
    torch.manual_seed(2)
    model = block.Model()
    sequences = [torch.randint(0, 64, (n,), device="cuda") for n in (37, 1, 80)]
    whole = torch.tensor([0, 37, 38, 118], device="cuda")
    want = model.serve(torch.cat(sequences), model.states(3), whole)
    # all but the last token as prompts (one of them empty), the last as a step
    heads = torch.tensor([0, 36, 36, 115], device="cuda")
    states = model.states(3)
    first = model.serve(torch.cat([s[:-1] for s in sequences]), states, heads)
    last = model.serve(torch.stack([s[-1] for s in sequences]), states)
    kept = torch.cat([torch.arange(0, 36), torch.arange(38, 117)]).cuda()
    # the same operations on the same values: what differs is the order of sums, and codes of 4 bits that fall to the other side
    assert (first.float() - want[kept].float()).norm() <= 0.02 * want.float().norm()
    assert (last.float() - want[whole[1:] - 1].float()).norm() <= 0.02 * want[whole[1:] - 1].float().norm()


def test_partial_gradients(block):
    from paper_1811_09736_amd import autograd
    q, k, v = (torch.randn(1, 20, 2, 64, device="cuda", dtype=torch.float16, requires_grad=True) for _ in range(3))
    state = torch.randn(1, 2, 64, 64, device="cuda", requires_grad=True)
    decay = torch.full((2,), -0.1, device="cuda")
    out, last = autograd.linear_attention(q, k, v, decay, state=state)
    last.sum().backward()                                       # only the last state is used
    assert (q.grad == 0).all() and (state.grad - torch.exp(torch.tensor(-2.0))).abs().max() < 1e-5 and k.grad.abs().sum() > 0
    x, w = torch.randn(4, 100, device="cuda", requires_grad=True), torch.randn(100, device="cuda", requires_grad=True)
    y, total = autograd.rms_norm(x, w, residual=torch.ones(4, 100, device="cuda"))
    total.sum().backward()                                      # only the sum is used
    assert torch.allclose(x.grad, torch.ones_like(x)) and (w.grad == 0).all()

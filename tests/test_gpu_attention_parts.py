"""How exact the derived operands of chunked linear attention are: what the header of the kernels claims, held tightly enough that a part less would show.

Bounds, relative to the sum of magnitudes of an output's terms.  Scores, and states as factors, are two parts: off by 2^-17 (bfloat16) or 2^-20 (binary16) each, one of the two in
each term, and sums of binary32 round by 2^-24 a product of 32; then one rounding to the type: u |want| + 2^-16 size.  (One part: 2^-9 or 2^-11 of a term.)  What is added to
states is off by 2^-21, their sums over few tokens by a few 2^-24: 2^-20 size.  (Two bfloat16 parts: 2^-17, one binary16 part: 2^-11.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_SPACING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


def definition(q, k, v, decay, s, scale):
    """[B, T, H, d] in 64 bits: out and the last states; differentiable."""
    q, k, v = (x.transpose(1, 2) for x in (q, k, v))
    t = torch.arange(q.shape[2], device=q.device, dtype=torch.float64)
    rel, a = t[:, None] - t[None, :], decay.double()[:, None, None]
    w = torch.where(rel >= 0, torch.exp(a * rel.clamp(min=0)), 0.0)
    front, behind = torch.exp(a * (t + 1)[:, None]), torch.exp(a * (len(t) - 1 - t)[:, None])
    out = scale * (torch.matmul(torch.matmul(q, k.transpose(2, 3)) * w, v) + torch.matmul(q * front, s))
    return out.transpose(1, 2), torch.matmul((k * behind).transpose(2, 3), v) + torch.exp(a * len(t)) * s


def inputs(seed, dtype, batch, tokens, heads, d):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    make = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    q, k, v, dout = (make(batch, tokens, heads, d).to(dtype) for _ in range(4))
    decay = -0.2 * torch.rand(heads, generator=gen, device="cuda")
    return q, k, v, dout, decay, make(batch, heads, d, d) * 3, make(batch, heads, d, d)


def check(got, want, size, u, more):
    off = (got.double() - want).abs() - u * want.abs() - more * size
    assert (off <= 0).all(), (off / size).max().item()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("batch,tokens,heads,d", [(40, 5, 2, 8), (40, 16, 2, 64), (8, 64, 4, 128), (4, 40, 2, 256), (1, 700, 2, 64)])
def test_parts(tcr, dtype, batch, tokens, heads, d):
    q, k, v, dout, decay, state, dfinal = inputs(d + tokens, dtype, batch, tokens, heads, d)
    u = HALF_SPACING[dtype]
    ins = [x.double().requires_grad_() for x in (q, k, v, state)]
    out, last = definition(*ins[:3], decay, ins[3], d ** -0.5)
    grads = torch.autograd.grad((out * dout.double()).sum() + (last * dfinal.double()).sum(), ins)
    big = [x.double().abs().requires_grad_() for x in (q, k, v, state)]
    size, last_size = definition(*big[:3], decay, big[3], d ** -0.5)
    sizes = torch.autograd.grad((size * dout.double().abs()).sum() + (last_size * dfinal.double().abs()).sum(), big)
    got, got_last = tcr.linear_attention(q, k, v, decay, state=state, final_state=True)
    check(got, out.detach(), size.detach(), u, 2.0 ** -16)
    dq, dk, dv, dstate = tcr.linear_attention_backward(dout, q, k, v, decay, state=state, dfinal=dfinal)
    for g, w, z in zip((dq, dk, dv), grads, sizes):
        check(g, w, z, u, 2.0 ** -16)
    if tokens <= 16:
        check(got_last, last.detach(), last_size.detach(), 0.0, 2.0 ** -20)
        check(dstate, grads[3], sizes[3], 0.0, 2.0 ** -20)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_states_of_few_products(tcr, dtype):
    # three products an entry, and nothing else in it: the parts of what is added
    q, k, v, dout, decay, _, _ = inputs(3, dtype, 64, 3, 4, 64)
    zeros = torch.zeros(64, 4, 64, 64, device="cuda", dtype=torch.float64)
    _, last = tcr.linear_attention(q, k, v, decay, final_state=True)
    want = definition(*(x.double() for x in (q, k, v)), decay, zeros, 0.125)[1]
    size = definition(*(x.double().abs() for x in (q, k, v)), decay, zeros, 0.125)[1]
    check(last, want, size, 0.0, 2.0 ** -20)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_small_values_beside_large_ones(tcr, dtype):
    # columns from 1 to 2^-12 beside one another, as features of a model have them: each one's states are as exact as the others'
    q, k, v, dout, decay, _, _ = inputs(4, dtype, 64, 3, 4, 64)
    v, dout = (((x.float() + 3.0 * x.float().sign()) * torch.exp2(-(torch.arange(64, device="cuda") % 13))).to(dtype) for x in (v, dout))
    zeros = torch.zeros(64, 4, 64, 64, device="cuda", dtype=torch.float64)
    _, last = tcr.linear_attention(q, k, v, decay, final_state=True)
    want = definition(*(x.double() for x in (q, k, v)), decay, zeros, 0.125)[1]
    size = definition(*(x.double().abs() for x in (q, k, v)), decay, zeros, 0.125)[1]
    check(last, want, size, 0.0, 2.0 ** -20)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_shared_heads_repeat(tcr, dtype):
    # binary32 outputs of each head, 16 bytes a store, all of them the same every time
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    make = lambda h: torch.randn(2, 1500, h, 128, generator=gen, device="cuda").to(dtype)  # noqa: E731
    q, k, v, dout = make(8), make(4), make(4), make(8)
    decay = -0.1 * torch.rand(8, generator=gen, device="cuda")
    want = tcr.linear_attention_backward(dout, q, k, v, decay)[:3]
    for _ in range(12):
        assert all(torch.equal(a, b) for a, b in zip(tcr.linear_attention_backward(dout, q, k, v, decay)[:3], want))

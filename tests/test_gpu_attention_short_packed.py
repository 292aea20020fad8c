"""Packed sequences that go token by token (two tokens or fewer on average): empty ones, single tokens, a long one among them, tokens in none; forwards, and backwards with a
state and the gradient of the last states.  Token strides that no chunk takes.  Tolerances as in test_gpu_attention.py: outputs and 16-bit gradients are rounded once, by u
of themselves, and sums of binary32 in front of it are off by 2^-20 of the magnitudes at most (300 tokens of 2^-24 each would be 2^-16 were they all rounded to one side;
magnitudes decay); states by 2^-19 of theirs."""
import ctypes

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


def make(gen, *shape, dtype=torch.float32, spread=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(dtype)


def run(q, k, v, decay, cuts, state, scale):
    """The recurrence in 64 bits; differentiable.  Rows outside the sequences: 0."""
    heads, group = q.shape[1], q.shape[1] // k.shape[1]
    lam = torch.exp(decay.double())[:, None, None]
    out, last = [torch.zeros(heads, v.shape[2], dtype=torch.float64, device=q.device)] * q.shape[0], []
    for n, (a, b) in enumerate(zip(cuts, cuts[1:])):
        s = state[n]
        for t in range(a, b):
            s = lam * s + k[t].repeat_interleave(group, 0)[:, :, None] * v[t].repeat_interleave(group, 0)[:, None, :]
            out[t] = scale * (q[t][:, :, None] * s).sum(1)
        last.append(s)
    return torch.stack(out), torch.stack(last)


def gradients(loss, ins):
    """(Zeros where no sequence has a token.)"""
    return [torch.zeros_like(x) if g is None else g for g, x in zip(torch.autograd.grad(loss, ins, allow_unused=True), ins)]


def near(got, want, size, u, more):
    off = (got.double() - want).abs() - (u * want.abs() + more * size + 1e-30)
    assert not torch.isnan(got).any() and (off <= 0).all(), (off.max().item(), (off > 0).sum().item())


CUTS = {"ones": list(range(0, 41)),
        "empties and gaps": [7, 7, 8, 8, 8, 10, 11, 11, 12, 14, 14, 15, 16, 18, 18],
        "a long one": [3] + [3 + i for i in range(1, 150)] + [300] + [300 + i for i in range(1, 12)],
        "none": [5, 5, 5, 5, 5, 5, 5, 5, 5, 5]}


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv,dk,dv", [(2, 2, 64, 64), (4, 2, 24, 72), (6, 1, 128, 16)])
@pytest.mark.parametrize("name", CUTS)
def test_short_packed_sequences(tcr, name, heads, kv, dk, dv, dtype):
    cuts = CUTS[name]
    tokens, count = cuts[-1] + 6, len(cuts) - 1
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens + heads)
    q, k, v = make(gen, tokens, heads, dk, dtype=dtype), make(gen, tokens, kv, dk, dtype=dtype), make(gen, tokens, kv, dv, dtype=dtype)
    decay = -torch.rand(heads, generator=gen, device="cuda") * 0.3
    state, dfinal, dout = make(gen, count, heads, dk, dv, spread=3.0), make(gen, count, heads, dk, dv), make(gen, tokens, heads, dv, dtype=dtype)
    offsets, u, scale = torch.tensor(cuts, device="cuda"), HALF_SPACING[dtype], dk ** -0.5

    ins = [x.double().requires_grad_() for x in (q, k, v, state)]
    want, last = run(*ins[:3], decay, cuts, ins[3], scale)
    grads = gradients((want * dout.double()).sum() + (last * dfinal.double()).sum(), ins)
    big = [x.double().abs().requires_grad_() for x in (q, k, v, state)]
    size, last_size = run(*big[:3], decay, cuts, big[3], scale)
    sizes = gradients((size * dout.double().abs()).sum() + (last_size * dfinal.double().abs()).sum(), big)

    room = torch.full((tokens + 2, heads, dv), 7.0, dtype=dtype, device="cuda")
    out = room[1:-1]
    got, got_last = tcr.linear_attention(q, k, v, decay, offsets=offsets, state=state, final_state=True, out=out)
    near(got, want.detach(), size.detach(), u, 2.0 ** -20)
    near(got_last, last.detach(), last_size.detach(), 0.0, 2.0 ** -19)
    assert (got[:cuts[0]] == 0).all() and (got[cuts[-1]:] == 0).all() and (room[0] == 7).all() and (room[-1] == 7).all()
    for g, w, z, bound in zip(tcr.linear_attention_backward(dout, q, k, v, decay, offsets=offsets, state=state, dfinal=dfinal), grads, sizes, (u, u, u, 0.0)):
        near(g, w, z, bound, 2.0 ** -20 if bound else 2.0 ** -19)
        if bound:
            assert (g[:cuts[0]] == 0).all() and (g[cuts[-1]:] == 0).all()


def test_tokens_in_the_other_order(tcr):
    # a negative token stride: the rows stand backwards in memory, which only the C call can say
    heads, tokens, d = 2, 90, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    q, k, v = (make(gen, tokens, heads, d, dtype=torch.float16) for _ in range(3))
    decay, state = torch.tensor([-0.1, -0.003], device="cuda"), torch.zeros(1, heads, d, d, device="cuda", dtype=torch.float64)
    want, last = run(*(x.flip(0).double() for x in (q, k, v)), decay, [0, tokens], state, 0.125)
    size, last_size = run(*(x.flip(0).double().abs() for x in (q, k, v)), decay, [0, tokens], state, 0.125)
    out, got_last = torch.empty_like(q), torch.empty(1, heads, d, d, device="cuda")
    a = tcr.AttentionShape()
    a.dtype, a.heads, a.kv_heads, a.dk, a.dv, a.sequences, a.tokens, a.scale = tcr.F16, heads, heads, d, d, 1, tokens, 0.125
    a.offsets, a.log_decay = None, decay.data_ptr()
    for s in (a.q_stride, a.k_stride, a.v_stride, a.o_stride):
        s[:] = [0, -heads * d, d]
    behind = (tokens - 1) * heads * d * 2
    st = tcr.raw().tcr_linear_attention(ctypes.byref(a), *(x.data_ptr() + behind for x in (q, k, v, out)), None, got_last.data_ptr(),
                                        torch.cuda.current_stream().cuda_stream)
    assert st == tcr.OK
    near(out.flip(0), want, size, HALF_SPACING[torch.float16], 2.0 ** -20)
    near(got_last, last, last_size, 0.0, 2.0 ** -19)


def test_far_apart_tokens(tcr):
    # a token stride beyond 2^23 elements, which no chunk's offsets hold
    heads, tokens, d = 1, 9, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(10)
    near_by = [make(gen, 1, tokens, heads, d, dtype=torch.bfloat16) for _ in range(3)]
    decay = torch.tensor([-0.1], device="cuda")
    stride = (1 << 23) + 8
    room = torch.empty(3 * d + tokens * stride, dtype=torch.bfloat16, device="cuda")
    far = [room[i * d:].as_strided((1, tokens, heads, d), (tokens * stride, stride, d, 1)) for i in range(3)]
    for f, x in zip(far, near_by):
        f.copy_(x)
    got, last = tcr.linear_attention(*far, decay, final_state=True)
    want, want_last = tcr.linear_attention(*near_by, decay, final_state=True)
    # (one token by token, one by a chunk: two roundings to bfloat16 of sums of binary32)
    assert ((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 2.0 ** -16 * want.float().abs().max()).all()
    assert (last - want_last).abs().max() <= 2.0 ** -19 * want_last.abs().max()

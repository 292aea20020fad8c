"""Gradients over arrays of more than 2^31 elements: 2^19 tokens of 4352 channels, bfloat16, against calls on their first and last tokens."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOKENS, CHANNELS, PART = 1 << 19, 4352, 4096


@pytest.fixture()
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    torch.cuda.synchronize()
    binding.release()
    torch.cuda.empty_cache()


def inputs():
    """One row of x for all tokens; gradients of the outputs at the first and the last PART tokens, 0 between them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(61)
    x = torch.randn(1, 1, CHANNELS, generator=gen, device="cuda").to(torch.bfloat16).expand(1, TOKENS, CHANNELS)
    dout = torch.zeros(1, TOKENS, CHANNELS, device="cuda", dtype=torch.bfloat16)
    for part in (slice(0, PART), slice(TOKENS - PART, TOKENS)):
        dout[:, part] = torch.randn(1, PART, CHANNELS, generator=gen, device="cuda").to(torch.bfloat16)
    assert dout.numel() > 1 << 31
    return gen, x, dout


def test_convolution(tcr):
    gen, x, dout = inputs()
    taps = torch.randn(CHANNELS, 4, generator=gen, device="cuda").to(torch.bfloat16)
    dx, dweight, _, _ = tcr.causal_conv_backward(dout, x, taps)
    first = tcr.causal_conv_backward(dout[:, :PART + 8].contiguous(), x[:, :PART + 8], taps)
    last = tcr.causal_conv_backward(dout[:, TOKENS - PART:], x[:, TOKENS - PART:], taps, state=x[:, :3].contiguous())
    half = TOKENS - PART
    assert torch.equal(dx[:, :PART + 8], first[0]) and torch.equal(dx[:, half:], last[0])
    assert torch.equal(dx[0, half - 3:half], last[3][0]) and (dx[:, PART + 8:half - 3] == 0).all()
    # all three rounded to bfloat16, and additions of 8192 terms, none larger than 1.1 |dout x|, in other orders
    want = first[1].float() + last[1].float()
    size = 1.1 * (dout[0, :PART].float().abs().sum(0) + dout[0, half:].float().abs().sum(0)) * x[0, 0].float().abs()
    room = 2.0 ** -8 * (first[1].float().abs() + last[1].float().abs() + want.abs()) + 2 * 8192 * 2.0 ** -24 * size[:, None]
    assert ((dweight.float() - want).abs() <= room).all()


def test_selective_scan(tcr):
    gen, x, dout = inputs()
    a = -torch.rand(CHANNELS, 4, generator=gen, device="cuda") - 0.1
    b = torch.randn(1, TOKENS, 1, 4, generator=gen, device="cuda").to(torch.bfloat16)
    dx, ddt, da, db, dc, *_ = tcr.selective_scan_backward(dout, x, x, a, b, b)
    half, mid = TOKENS - PART, TOKENS - 6 * PART
    # Steps are softplus of at least -4 or so, 0.018, and rates 0.1 and more: over 20480 tokens all dies out, e^-37.  So the first tokens are a call of their own, the last ones
    # go on from the states in front of them, and what they hand back lies in the 20480 in front of them.
    assert float(x.min()) > -4.5
    states = lambda to: tcr.selective_scan(x[:, :to], x[:, :to], a, b[:, :to], b[:, :to], final_state=True)[1]  # noqa: E731
    first = tcr.selective_scan_backward(dout[:, :PART], x[:, :PART], x[:, :PART], a, b[:, :PART], b[:, :PART])
    last = tcr.selective_scan_backward(dout[:, half:], x[:, half:], x[:, half:], a, b[:, half:], b[:, half:], state=states(half))
    between = tcr.selective_scan_backward(dout[:, mid:half], x[:, mid:half], x[:, mid:half], a, b[:, mid:half], b[:, mid:half], state=states(mid), dfinal=last[8])
    for i, got in ((0, dx), (1, ddt), (3, db), (4, dc)):
        got = got.flatten(2)
        for part, want in ((slice(0, PART), first[i]), (slice(mid, half), between[i]), (slice(half, TOKENS), last[i])):
            # Of every token: two roundings to bfloat16, 2^-8 each, and binary32 sums in other chunks -- 8 roundings a token for a hundred tokens, 2^-14, independent from channel to channel.
            off = (got[:, part].float() - want.flatten(2).float()).norm(dim=-1)
            assert (off <= 2.0 ** -6 * want.flatten(2).float().norm(dim=-1) + 2.0 ** -100).all(), i
    # (up to 4096 partial sums a line, one behind the other: 2^-12)
    want = first[2] + between[2] + last[2]
    assert (da - want).norm() <= 2.0 ** -12 * want.norm()

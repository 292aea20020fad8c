"""Arrays of more than 2^31 elements through the convolution, the scan and the norm: 2^19 tokens of 4352 channels, bfloat16."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOKENS, CHANNELS = 1 << 19, 4352


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    torch.cuda.empty_cache()


def test_beyond_32_bits(tcr):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    # one row for all tokens; b and c differ
    x = torch.randn(1, 1, CHANNELS, generator=gen, device="cuda").to(torch.bfloat16).expand(1, TOKENS, CHANNELS)
    a = -torch.rand(CHANNELS, 4, generator=gen, device="cuda") - 0.1
    b = torch.randn(1, TOKENS, 1, 4, generator=gen, device="cuda").to(torch.bfloat16)
    out, last = tcr.selective_scan(x, x, a, b, b, final_state=True)
    assert out.numel() > 1 << 31
    # the last 4096 tokens once more, from the states of those in front
    half = TOKENS - 4096
    _, state = tcr.selective_scan(x[:, :half], x[:, :half], a, b[:, :half], b[:, :half], final_state=True)
    tail, end = tcr.selective_scan(x[:, half:], x[:, half:], a, b[:, half:], b[:, half:], state=state, final_state=True)
    # the same sums in other chunks: a step of bfloat16 where a rounding falls to the other side
    assert ((out[:, half:].float() - tail.float()).abs() <= 2.0 ** -7 * tail.float().abs() + 1e-5).all()
    assert (last - end).norm() <= 2.0 ** -19 * end.norm()
    taps = torch.ones(CHANNELS, 4, device="cuda", dtype=torch.bfloat16)
    h = tcr.causal_conv(out, taps, activation=None)
    for at in (4, half, TOKENS):
        want = ((out[:, at - 4].float() + out[:, at - 3].float()) + out[:, at - 2].float()) + out[:, at - 1].float()
        assert torch.equal(h[:, at - 1], want.to(torch.bfloat16))
    del h
    want = sum(float(part.double().square().sum()) for part in out[0].split(1 << 15)) ** 0.5
    assert abs(float(tcr.gradient_norm([out])) - want) <= 2.0 ** -23 * want

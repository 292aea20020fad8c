"""States that decay slowly over many chunks and blocks.

Tolerance.  A state is multiplied by its decay once a chunk (a block), rounded each time by at most half a spacing, 2^-24 of itself and of either sign: a
deviation of 2^-23 / sqrt(12) for each, so 512 of them come to 2^-20.3 and 2^-18 is five deviations.  The decay itself must not add an error that is
the same every time: 512 roundings of 2^-25 to one side would be 2^-16."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# natural logarithms whose 64-token decay is rounded by much of half a spacing
SLOW = [-0.9 * 2.0 ** -15, -(2.0 ** -18), -(2.0 ** -12), -(2.0 ** -13)]


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


def near(got, want, size):
    off = (got.double() - want).abs() / size
    assert off.max().item() <= 2.0 ** -18, off.max().item()


def small(gen, *shape, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * 1e-3).to(dtype)


def sums(a, b, log_decay, reverse):
    """(S, sum of magnitudes) behind [tokens, heads, 8] rows: S = sum over t of exp(log_decay steps) a_t b_t^T, in 64 bits."""
    t = torch.arange(a.shape[0], device="cuda", dtype=torch.float64)
    weight = torch.exp(log_decay.double()[:, None] * ((t + 1) if reverse else (len(t) - 1 - t)))[..., None]
    a, b = a.double().transpose(0, 1).contiguous(), b.double().transpose(0, 1).contiguous()
    at = (a * weight).transpose(1, 2).contiguous()
    return torch.matmul(at, b), torch.matmul(at.abs(), b.abs())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens,heads,decays", [(32768, 1024, SLOW),                       # as many heads as fill the chip: a sequence in one block
                                                 (262144, 2, [-0.9 * 2.0 ** -15, -0.7 * 2.0 ** -18]),    # two heads in 256 blocks
                                                 (262144, 2, [-0.9 * 2.0 ** -16, -(2.0 ** -15)]),
                                                 (4096, 32, SLOW)])                         # blocks that add up the states in front themselves
def test_slow_decays(tcr, dtype, tokens, heads, decays):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens + heads)
    q, k, v, dout = (small(gen, 1, tokens, heads, 8, dtype=dtype) for _ in range(4))
    decay = torch.tensor(decays, device="cuda").repeat(-(-heads // len(decays)))[:heads].contiguous()
    state, dfinal = (torch.randn(1, heads, 8, 8, generator=gen, device="cuda") * 3 for _ in range(2))
    left = torch.exp(decay.double() * tokens)[None, :, None, None]
    out, last = tcr.linear_attention(q, k, v, decay, state=state, final_state=True)
    del out
    want, size = sums(k[0], v[0], decay, False)
    near(last, want + left * state.double(), size + left * state.double().abs())
    dstate = tcr.linear_attention_backward(dout, q, k, v, decay, scale=1.0, state=state, dfinal=dfinal)[3]
    want, size = sums(q[0], dout[0], decay, True)
    near(dstate, want + left * dfinal.double(), size + left * dfinal.double().abs())

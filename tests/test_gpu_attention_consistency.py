"""What gradients of linear attention may depend on: not on which of their results are asked for, and as scans they are the forward pass's."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("batch,tokens,heads,kv", [(2, 700, 4, 4), (1, 3000, 4, 2), (16, 300, 8, 8)])
def test_gradients_do_not_depend_on_whether_a_state_is_given(tcr, dtype, batch, tokens, heads, kv):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens)
    make = lambda h: torch.randn(batch, tokens, h, 128, generator=gen, device="cuda").to(dtype)  # noqa: E731
    q, k, v, dout = make(heads), make(kv), make(kv), make(heads)
    decay = -0.05 * torch.rand(heads, generator=gen, device="cuda")
    without = tcr.linear_attention_backward(dout, q, k, v, decay)
    zeros = torch.zeros(batch, heads, 128, 128, device="cuda")
    given = tcr.linear_attention_backward(dout, q, k, v, decay, state=zeros, dfinal=zeros.clone())
    # (the states in front add zeros; nothing else is different)
    for a, b in zip(without[:3], given[:3]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("batch,tokens", [(2, 200), (1, 5000), (64, 300)])
def test_the_gradient_of_queries_is_an_attention(tcr, dtype, batch, tokens):
    # dq is the attention of (dout, v, k): the same scan, to the same precision
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens)
    q, k, v, dout = (torch.randn(batch, tokens, 4, 64, generator=gen, device="cuda").to(dtype) for _ in range(4))
    decay = -0.05 * torch.rand(4, generator=gen, device="cuda")
    dq = tcr.linear_attention_backward(dout, q, k, v, decay, scale=0.125)[0]
    assert torch.equal(dq, tcr.linear_attention(dout, v, k, decay, scale=0.125))

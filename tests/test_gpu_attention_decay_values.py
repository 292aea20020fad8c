"""Decays that are no number: their head's results say so, and no other head's change."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 2, 40, 300, 3000])
def test_a_decay_that_is_none_shows(tcr, bad, dtype, tokens):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(tokens)
    q, k, v, dout = (torch.randn(2, tokens, 3, 64, generator=gen, device="cuda").to(dtype) for _ in range(4))
    state = torch.randn(2, 3, 64, 64, generator=gen, device="cuda")
    decay = torch.tensor([-0.1, -0.02, -0.003], device="cuda")
    spoilt = decay.clone()
    spoilt[1] = bad
    want = tcr.linear_attention(q, k, v, decay, state=state, final_state=True)
    out, last = tcr.linear_attention(q, k, v, spoilt, state=state, final_state=True)
    grads = tcr.linear_attention_backward(dout, q, k, v, decay, state=state)
    got = tcr.linear_attention_backward(dout, q, k, v, spoilt, state=state)
    others = [0, 2]
    assert torch.equal(out[:, :, others], want[0][:, :, others]) and torch.equal(last[:, others], want[1][:, others])
    assert not torch.isfinite(out[:, :, 1]).any() and not torch.isfinite(last[:, 1]).any()
    for a, b in zip(got[:3], grads):
        assert torch.equal(a[:, :, others], b[:, :, others])
    assert torch.equal(got[3][:, others], grads[3][:, others])
    if tokens > 1:                                  # (dq of the first token has the decayed state in it, dk and dv of the last token no decay)
        assert not torch.isfinite(got[1][:, 0, 1]).any() and not torch.isfinite(got[2][:, 0, 1]).any()
    assert not torch.isfinite(got[0][:, :, 1]).any() and not torch.isfinite(got[3][:, 1]).any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_step(tcr, bad):
    q, k, v = (torch.randn(5, 2, 64, device="cuda").half() for _ in range(3))
    state = torch.randn(5, 2, 64, 64, device="cuda")
    good, spoilt = torch.tensor([-0.1, -0.1], device="cuda"), torch.tensor([bad, -0.1], device="cuda")
    a, b = state.clone(), state.clone()
    want, got = tcr.linear_attention_step(q, k, v, good, a), tcr.linear_attention_step(q, k, v, spoilt, b)
    assert torch.equal(got[:, 1], want[:, 1]) and torch.equal(a[:, 1], b[:, 1])
    assert not torch.isfinite(got[:, 0]).any() and not torch.isfinite(b[:, 0]).any()

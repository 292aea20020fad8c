"""Outputs of linear attention among its inputs' memory, but not in their place, are right; in their place they are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


@pytest.mark.parametrize("d", [64, 256])
@pytest.mark.parametrize("tokens", [1, 3, 200])
def test_outputs_beside_the_inputs_in_one_projections_rows(tcr, tokens, d):
    decay = torch.tensor([-0.1, -0.01], device="cuda")
    for dtype in (torch.float16, torch.bfloat16):
        rows = torch.randn(2, tokens, 4, 2, d, device="cuda").to(dtype)
        q, k, v, out = rows.unbind(2)
        want = tcr.linear_attention(q.contiguous(), k.contiguous(), v.contiguous(), decay)
        assert tcr.linear_attention(q, k, v, decay, out=out) is out and torch.equal(out, want)
        parts = torch.randn(4, 2, tokens, 2, d, device="cuda").to(dtype)          # one behind the other
        q, k, v, out = parts
        want = tcr.linear_attention(q, k, v, decay)
        assert torch.equal(tcr.linear_attention(q, k, v, decay, out=out), want)
        state = torch.randn(2, 2, d, d, device="cuda")
        want = tcr.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state.clone())
        assert torch.equal(tcr.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state, out=out[:, 0]), want)


def test_outputs_in_an_inputs_place(tcr):
    decay = torch.tensor([-0.1, -0.01], device="cuda")
    q, k, v = (torch.randn(2, 30, 2, 64, device="cuda").half() for _ in range(3))
    state = torch.randn(2, 2, 64, 64, device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        for place in (q, k, v):
            for call in (lambda: tcr.linear_attention(q, k, v, decay, out=place, stream=stream),
                         lambda: tcr.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state, out=place[:, 0], stream=stream)):
                with pytest.raises(tcr.TcrError) as e:
                    call()
                assert e.value.status == tcr.ERR_INVALID_ARG

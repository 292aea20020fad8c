"""Tensors that calls write in place count as changed: autograd notices one that it has kept."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


def streams():
    """The current stream as every call takes it, and named (which goes another way through the binding)."""
    return None, torch.cuda.current_stream()


def rows(*shape):
    return torch.randn(*shape, device="cuda").half()


def test_a_state_stepped_in_place_is_noticed(tcr):
    from paper_1811_09736_amd import autograd
    decay = torch.full((2,), -0.1, device="cuda")
    for stream in streams():
        for place in ("state", "new_state", "out"):
            q, k, v = (rows(1, 20, 2, 64).requires_grad_() for _ in range(3))
            state = torch.randn(1, 2, 64, 64, device="cuda")
            out, last = autograd.linear_attention(q, k, v, decay, state=state)
            q1, k1, v1 = (rows(1, 2, 64) for _ in range(3))
            if place == "state":
                tcr.linear_attention_step(q1, k1, v1, decay, state, stream=stream)
            elif place == "new_state":
                tcr.linear_attention_step(q1, k1, v1, decay, torch.zeros_like(state), new_state=state, stream=stream)
            else:
                tcr.linear_attention(*(rows(1, 20, 2, 64) for _ in range(3)), decay, out=q.detach(), stream=stream)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                out.sum().backward()


def test_versions(tcr):
    decay = torch.full((2,), -0.1, device="cuda")
    q, k, v = (rows(3, 2, 64) for _ in range(3))
    for stream in streams():
        state, new, out = torch.zeros(3, 2, 64, 64, device="cuda"), torch.zeros(3, 2, 64, 64, device="cuda"), rows(3, 2, 64)
        ins = (q, k, v, decay)
        before = [x._version for x in (*ins, state, new, out)]
        tcr.linear_attention_step(q, k, v, decay, state, new_state=new, out=out, stream=stream)
        assert [x._version for x in (*ins, state, new, out)] == [*before[:5], before[5] + 1, before[6] + 1]
        tcr.linear_attention_step(q, k, v, decay, state, stream=stream)
        assert state._version == before[4] + 1


def test_tensors_without_versions(tcr):
    # made in inference mode: nothing to count, inside and outside of it
    with torch.inference_mode():
        decay = torch.full((2,), -0.1, device="cuda")
        q, k, v = (rows(3, 2, 64) for _ in range(3))
        state = torch.zeros(3, 2, 64, 64, device="cuda")
        for stream in streams():
            tcr.linear_attention_step(q, k, v, decay, state, stream=stream)
    for stream in streams():
        tcr.linear_attention_step(q, k, v, decay, state, out=torch.empty_like(q), stream=stream)
    torch.cuda.synchronize()
    assert torch.isfinite(state).all() and state.abs().sum() > 0

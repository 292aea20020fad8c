"""What the differentiable forms refuse, which needs no GPU: it is checked in front of everything else."""
import pytest
import torch

from paper_1811_09736_amd import autograd


def inputs():
    q, k, v = (torch.zeros(1, 4, 2, 8, dtype=torch.float16, requires_grad=True) for _ in range(3))
    return q, k, v, torch.full((2,), -0.1)


def test_a_decay_that_wants_a_gradient_is_refused():
    q, k, v, decay = inputs()
    learned = decay.clone().requires_grad_()
    for wanted in (learned, learned * 2.0, torch.nn.Parameter(decay)):
        with pytest.raises(ValueError, match="log_decay"):
            autograd.linear_attention(q, k, v, wanted)
    # without gradients, or detached, it goes on (here as far as to the tensors that are not on a GPU)
    with torch.no_grad(), pytest.raises(TypeError, match="q must be"):
        autograd.linear_attention(q, k, v, learned)
    with pytest.raises(TypeError, match="q must be"):
        autograd.linear_attention(q, k, v, learned.detach())

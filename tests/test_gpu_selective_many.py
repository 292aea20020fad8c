"""Gradients of the selective scan carried over more chunks than one round takes, 64, in chunks of 32 tokens.  Bounds as in test_gpu_selective.py's test of chunks of 8."""
import pytest
import torch

from test_gpu_selective import check_grads, grads_of, make, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    binding.check_device_flags()


@pytest.mark.parametrize("states,groups", [(16, 1), (32, 2), (40, 1)], ids=str)
@pytest.mark.parametrize("bounds", [None, [0, 3, 2060, 2100, 2100, 2190], [70, 2150]], ids=str)
def test_more_than_one_round(tcr, states, groups, bounds):
    tokens = 2200
    lead, count = ((1, tokens), 1) if bounds is None else ((tokens,), len(bounds) - 1)
    v = make(torch.float32, lead, 20, states, groups, state=count, seed=51)
    offsets = None if bounds is None else torch.tensor(bounds, device="cuda")
    dout, dfinal = torch.randn(*lead, 20, device="cuda"), torch.randn(count, 20, states, device="cuda")
    got = grads_of(tcr, v, dout, offsets, dfinal)
    want, large = (reference(**v, softplus=True, offsets=offsets, dout=dout, dfinal=dfinal, large=m) for m in (False, True))
    check_grads(got, want, large, tokens, tokens, v)
    for name in ("dx", "ddt", "db", "dc", "dgate", "dstate"):
        # errors of independent roundings that die out within some hundred tokens
        assert (got[name].double() - want[name]).norm() <= 2.0 ** -19 * want[name].norm(), name

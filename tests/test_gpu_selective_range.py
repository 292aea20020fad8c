"""The selective scan and its gradients where the factor over a chunk of tokens leaves binary32's range and the states and gradients themselves do not: the recurrence goes
token by token, with factors that are in range, and its results must not depend on how the tokens are cut.

Tolerances: as in test_gpu_selective.py, (roundings a token) * tokens * 2^-24 of every term's magnitude.  A token's factor exp(e) carries the roundings of its argument -- of the constant, of the
rate and of the product, and of sums of steps, which are exact here -- as often as its exponent e says: 4 |e| beside the 8 of the recurrence, backwards as often again."""
import pytest
import torch

from test_gpu_selective import check, make, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    binding.check_device_flags()


def inputs(tokens, channels, states, lead=1):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(31)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return {"x": rand(lead, tokens, channels), "dt": torch.zeros(lead, tokens, channels, device="cuda"), "a": torch.ones(channels, states, device="cuda"),
            "b": rand(lead, tokens, 1, states), "c": rand(lead, tokens, 1, states), "skip": rand(channels), "gate": None, "dt_bias": None, "state": None}


def forward(tcr, v, each):
    out, last = tcr.selective_scan(v["x"], v["dt"], v["a"], v["b"], v["c"], skip=v["skip"], softplus=False, state=v["state"], final_state=True)
    want, large = (reference(**v, softplus=False, offsets=None, large=m) for m in (False, True))
    assert torch.isfinite(want[0]).all() and float(want[1].abs().max()) < 2.0 ** 126
    tokens, states = v["x"].shape[1], v["a"].shape[1]
    terms = tokens * (8 + 4 * each) + states + 16
    check(out, want[0], large[0], terms, "out")
    check(last, want[1], large[1], terms, "states")


def backward(tcr, v, each, dout, dfinal=None):
    got = tcr.selective_scan_backward(dout, v["x"], v["dt"], v["a"], v["b"], v["c"], skip=v["skip"], softplus=False, state=v["state"], dfinal=dfinal)
    want, large = (reference(**v, softplus=False, offsets=None, dout=dout, dfinal=dfinal, large=m) for m in (False, True))
    tokens, states = v["x"].shape[1], v["a"].shape[1]
    terms = 2 * tokens * (8 + 4 * each) + states + 32 + v["x"].shape[2] + tokens
    for name, g in zip(("dx", "ddt", "da", "db", "dc", "dskip", "dgate", "dbias", "dstate"), got):
        if g is not None:
            assert torch.isfinite(want[name]).all() and float(want[name].abs().max()) < 2.0 ** 126, name
            check(g, want[name], large[name], terms, name)


@pytest.mark.parametrize("states", [1, 7, 16, 32, 64])
@pytest.mark.parametrize("tokens,step,near", [(4096, 2.0, 20), (2500, 8.0, 5), (8192, 0.75, 60)], ids=str)
def test_growing_factors_and_nothing_to_grow(tcr, states, tokens, step, near):
    """exp(step) a token, over chunks far beyond the range; inputs are 0 but for the last tokens."""
    v = inputs(tokens, 20, states)
    v["dt"] += step
    v["x"][:, :-near] = 0
    forward(tcr, v, step)


@pytest.mark.parametrize("states", [1, 7, 16, 32, 64])
@pytest.mark.parametrize("period,step", [(64, 2.0), (100, 1.25)], ids=str)
def test_states_that_shrink_far_and_grow_again(tcr, states, period, step):
    """1e30 e^-128 and back, one way or both in each chunk."""
    v = inputs(4000, 20, states)
    v["dt"] += torch.where(torch.arange(4000, device="cuda") // period % 2 == 0, -step, step)[None, :, None]
    v["x"].zero_()
    v["state"] = torch.full((1, 20, states), 1e30, device="cuda")
    forward(tcr, v, step)


@pytest.mark.parametrize("states", [1, 7, 16, 32, 64])
@pytest.mark.parametrize("tokens,step,near", [(700, 2.0, 20), (700, 8.0, 5), (2100, 0.75, 60)], ids=str)
def test_gradients_that_grow_backwards(tcr, states, tokens, step, near):
    """Gradients of the outputs are 0 but for the first tokens, inputs 0 but for the last ones."""
    v = inputs(tokens, 20, states)
    v["dt"] += step
    v["x"][:, :-near] = 0
    dout = torch.randn(1, tokens, 20, device="cuda")
    dout[:, near:] = 0
    backward(tcr, v, step, dout)


@pytest.mark.parametrize("states", [1, 7, 16, 32, 64])
@pytest.mark.parametrize("half,step", [(16, 8.0), (20, 6.0)], ids=str)
def test_gradients_that_grow_and_shrink_again(tcr, states, half, step):
    """Within a chunk of 32 tokens e^-128 and e^128; gradients of 1e-30 that reach 1e22, states of 1e25 that reach 1e-31."""
    tokens = 8 * half
    v = inputs(tokens, 20, states)
    v["dt"] += torch.where(torch.arange(tokens, device="cuda") // half % 2 == 0, -step, step)[None, :, None]
    v["x"].zero_()
    v["state"] = torch.full((1, 20, states), 1e25, device="cuda")
    dout = torch.zeros(1, tokens, 20, device="cuda")
    dout[:, 2 * half - 1::2 * half] = 1e-30 * torch.randn(1, 4, 20, device="cuda")
    backward(tcr, v, step, dout)


GAPS = [3, 3, 10, 11, 11, 11, 97, 130, 130, 257, 300]


@pytest.mark.parametrize("states,groups", [(3, 1), (8, 2), (16, 1), (32, 1), (64, 2)], ids=str)
@pytest.mark.parametrize("final", [True, False], ids=["final", "none"])
def test_packed_steps_of_both_signs(tcr, states, groups, final):
    v = make(torch.float32, (311,), 40, states, groups, bias=False, state=10, seed=33)     # (with a bias of the steps states would drift out of the range: 1e50)
    v["dt"] = (v["dt"] * 0.25).contiguous()
    offsets = torch.tensor(GAPS, device="cuda")
    dout, dfinal = torch.randn(311, 40, device="cuda"), torch.randn(10, 40, states, device="cuda") if final else None
    got = tcr.selective_scan_backward(dout, v["x"], v["dt"], v["a"], v["b"], v["c"], skip=v["skip"], gate=v["gate"], softplus=False, offsets=offsets, state=v["state"],
                                      dfinal=dfinal)
    want, large = (reference(**v, softplus=False, offsets=offsets, dout=dout, dfinal=dfinal, large=m) for m in (False, True))
    # 127 tokens of the longest sequence, exponents of up to 4; sums over 20 or 40 channels or 297 tokens
    for name, g in zip(("dx", "ddt", "da", "db", "dc", "dskip", "dgate", "dbias", "dstate"), got):
        if g is None:
            continue
        assert float(want[name].abs().max()) < 2.0 ** 126, name
        check(g, want[name], large[name], 2 * 127 * (8 + 4 * 4) + states + 32 + 300, name)

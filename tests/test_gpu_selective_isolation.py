"""Gradients of packed sequences: an infinity or NaN of one sequence stays in it, as in the outputs -- the gradients of the others are the same bits as without it."""
import pytest
import torch

from test_gpu_selective import make

pytestmark = pytest.mark.gpu

# Every bound behind the first stands in the midst of a chunk of 8, 16 and 32 tokens, behind chunks of the same sequence.
BOUNDS = [0, 43, 61, 77, 120]
HIT = 1                                        # the sequence that is hit, at its third token


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    binding.check_device_flags()


def gradients(tcr, v, dout, dfinal, offsets):
    got = tcr.selective_scan_backward(dout, v["x"], v["dt"], v["a"], v["b"], v["c"], skip=v["skip"], gate=v["gate"], dt_bias=v["dt_bias"], offsets=offsets, state=v["state"],
                                      dfinal=dfinal)
    return dict(zip(("dx", "ddt", "da", "db", "dc", "dskip", "dgate", "dbias", "dstate"), got))


def same_in_the_others(got, clean):
    of_token = torch.ones(BOUNDS[-1], dtype=torch.bool, device="cuda")
    of_token[BOUNDS[HIT]:BOUNDS[HIT + 1]] = False
    for name in ("dx", "ddt", "db", "dc", "dgate"):
        assert torch.isfinite(clean[name]).all(), name
        assert torch.equal(got[name][of_token], clean[name][of_token]), name
    others = [i for i in range(len(BOUNDS) - 1) if i != HIT]
    assert torch.equal(got["dstate"][others], clean["dstate"][others])


@pytest.mark.parametrize("dtype,channels,states,groups", [(torch.float32, 20, 16, 1), (torch.bfloat16, 24, 3, 2), (torch.float16, 33, 40, 1), (torch.float32, 70, 8, 1),
                                                          (torch.bfloat16, 40, 32, 1)], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf")], ids=str)
@pytest.mark.parametrize("name", ["dout", "x", "dt", "b", "c", "gate", "state", "dfinal"])
def test_what_is_not_finite_stays_in_its_sequence(tcr, dtype, channels, states, groups, value, name):
    v = {k: t.clone() for k, t in make(dtype, (BOUNDS[-1],), channels, states, groups, state=len(BOUNDS) - 1, seed=21).items()}
    v["dout"] = torch.randn(BOUNDS[-1], channels, device="cuda").to(dtype)
    v["dfinal"] = torch.randn(len(BOUNDS) - 1, channels, states, device="cuda")
    offsets = torch.tensor(BOUNDS, device="cuda")
    clean = gradients(tcr, v, v["dout"], v["dfinal"], offsets)
    v[name][HIT if name in ("state", "dfinal") else BOUNDS[HIT] + 2] = value           # (of all channels and states)
    got = gradients(tcr, v, v["dout"], v["dfinal"], offsets)
    hit = slice(BOUNDS[HIT], BOUNDS[HIT + 1])
    assert not all(torch.isfinite(got[k][hit]).all() for k in ("dx", "ddt", "db", "dc", "dgate"))
    same_in_the_others(got, clean)


def test_factors_beyond_the_range_stay_in_their_sequence(tcr):
    """A step whose factor is infinite: exp(500 / 2), of a state that grows."""
    v = {k: t.clone() for k, t in make(torch.float32, (BOUNDS[-1],), 20, 16, state=len(BOUNDS) - 1, seed=22).items()}
    v["a"][:, 5] = 0.5
    v["dt"] -= 4                                # (steps of the order of 1/50: the states that grow stay in range)
    dout, dfinal, offsets = torch.randn(BOUNDS[-1], 20, device="cuda"), torch.randn(len(BOUNDS) - 1, 20, 16, device="cuda"), torch.tensor(BOUNDS, device="cuda")
    clean = gradients(tcr, v, dout, dfinal, offsets)
    v["dt"][BOUNDS[HIT] + 2, 3] = 500.0
    got = gradients(tcr, v, dout, dfinal, offsets)
    assert not torch.isfinite(got["ddt"][BOUNDS[HIT]:BOUNDS[HIT + 1], 3]).all()
    same_in_the_others(got, clean)

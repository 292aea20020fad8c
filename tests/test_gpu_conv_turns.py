"""Gradients of the convolution where a thread takes more than one run of tokens: a workspace for one sum, and more runs than workgroups.  Bounds as in test_gpu_conv.py."""
import pytest
import torch

from test_gpu_conv import check, make, reference

pytestmark = pytest.mark.gpu
NAMES = ("dx", "dweight", "dbias", "dstate")


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    binding.set_workspace(None)


def compare(got, x, w, bias, act, offsets, state, dout, dfinal, tokens):
    want, large = (reference(x, w, bias, act, offsets, state, dout, dfinal, large=m) for m in (False, True))
    for name, g in zip(NAMES, got):
        if g is not None:
            check(g, want[name], large[name], 40 + (tokens if name in ("dweight", "dbias") else 0), name)


@pytest.mark.parametrize("dtype,channels,width", [(torch.float32, 70, 4), (torch.bfloat16, 24, 3), (torch.float16, 1033, 4), (torch.float32, 300, 2)], ids=str)
@pytest.mark.parametrize("packed", [False, True], ids=["dense", "packed"])
@pytest.mark.parametrize("sums", [1, 3])
def test_in_a_workspace_for_few_sums(tcr, dtype, channels, width, packed, sums):
    lead = (700,) if packed else (3, 233)
    bounds = [0, 1, 130, 130, 131, 600, 690]
    count = len(bounds) - 1 if packed else 3
    offsets = torch.tensor(bounds, device="cuda") if packed else None
    x, w, bias, state = make(dtype, lead, channels, width, True, count, seed=41)
    dout, dfinal = torch.randn(*lead, channels, device="cuda").to(dtype), torch.randn(count, width - 1, channels, device="cuda").to(dtype)
    given = dict(bias=bias, offsets=offsets, state=state, dfinal=dfinal)
    usual = tcr.causal_conv_backward(dout, x, w, **given)
    each = 4 * (width + 1) * channels          # bytes of a sum; the buffer's halves are multiples of 256
    area = -(-sums * each // 256) * 256
    assert area < (sums + 1) * each
    tcr.set_workspace(torch.empty(256 + 2 * area, dtype=torch.uint8, device="cuda"))
    try:
        got = tcr.causal_conv_backward(dout, x, w, **given)
        again = tcr.causal_conv_backward(dout, x, w, **given)
    finally:
        tcr.set_workspace(None)
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    assert torch.equal(got[0], usual[0]) and torch.equal(got[3], usual[3])
    compare(got, x, w, bias, True, offsets, state, dout, dfinal, 699)


def test_a_workspace_for_no_sum(tcr):
    x, w, bias, _ = make(torch.float32, (2, 50), 300, 4, True, None, seed=42)
    tcr.set_workspace(torch.empty(256 + 2 * 4096, dtype=torch.uint8, device="cuda"))             # 6000 bytes are one
    try:
        with pytest.raises(tcr.TcrError) as e:
            tcr.causal_conv_backward(x.contiguous(), x, w, bias=bias)
        assert e.value.status == tcr.ERR_WORKSPACE
    finally:
        tcr.set_workspace(None)


@pytest.mark.parametrize("dtype,width", [(torch.bfloat16, 4), (torch.float32, 4), (torch.float16, 2)], ids=str)
def test_more_runs_than_workgroups(tcr, dtype, width):
    """768 slabs of 256 channels, one workgroup each, four runs at a time: 3 sequences of 20 tokens are two runs each."""
    channels = 768 * 256
    x, w, bias, state = make(dtype, (3, 20), channels, width, True, 3, seed=43)
    dout = torch.randn(3, 20, channels, device="cuda").to(dtype)
    got = tcr.causal_conv_backward(dout, x, w, bias=bias, state=state)
    compare(got, x, w, bias, True, None, state, dout, None, 60)

"""The short causal convolution against its definition in 64 bits.  Sums of at most five products in binary32 and an activation of a few roundings: 32 * 2^-24 of the terms' magnitudes
(silu has a slope of at most 1.1), then half a step of the type; sums over tokens one rounding for each addition.  Last states are copies."""
import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -24
GAPS = [3, 3, 10, 11, 13, 13, 97, 130, 130, 257, 300]        # of 311 tokens


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    yield binding
    binding.check_device_flags()


def spans(x, offsets):
    if offsets is None:
        return [(i, slice(None)) for i in range(x.shape[0])]
    o = offsets.tolist()
    return [(slice(o[i], o[i + 1]),) for i in range(len(o) - 1)]


def reference(x, weight, bias, act, offsets, state, dout=None, dfinal=None, large=False):
    size = (lambda v: v.abs()) if large else (lambda v: v)
    channels, width = weight.shape
    x, w = x.double(), weight.double()
    bias = torch.zeros(channels, device=x.device, dtype=torch.float64) if bias is None else bias.double()
    parts = spans(x, offsets)
    out, last = torch.zeros_like(x), torch.zeros(len(parts), width - 1, channels, device=x.device, dtype=torch.float64)
    grads = {"dx": torch.zeros_like(x), "dweight": torch.zeros_like(w), "dbias": torch.zeros_like(bias), "dstate": torch.zeros_like(last)}
    for i, at in enumerate(parts):
        front = state[i].double() if state is not None else torch.zeros_like(last[i])
        full = torch.cat([front, x[at]])
        length = full.shape[0] - (width - 1)
        last[i] = full[length:]
        s = sum(full[j:j + length] * w[:, j] for j in range(width)) + bias
        sure = sum((full[j:j + length] * w[:, j]).abs() for j in range(width)) + bias.abs()
        z = 1 / (1 + torch.exp(-s))
        out[at] = sure if large else s * z if act else s
        if dout is None:
            continue
        # (large: the slope's two terms, and their own slope of at most 1/2 times the error of s)
        ds = size(dout[at].double())
        if act:
            ds = ds * ((z + s.abs() * z * (1 - z) + 0.5 * sure) if large else (z + s * z * (1 - z)))
        full = size(full)
        dfull = torch.zeros_like(full)
        for j in range(width):
            dfull[j:j + length] += ds * size(w[:, j])
            grads["dweight"][:, j] += (ds * full[j:j + length]).sum(0)
        if dfinal is not None:
            dfull[length:] += size(dfinal[i].double())
        grads["dx"][at], grads["dstate"][i] = dfull[width - 1:], dfull[:width - 1]
        grads["dbias"] += ds.sum(0)
    return (out, last) if dout is None else grads


def check(got, want, large, terms, name):
    half = 0.0 if got.dtype == torch.float32 else torch.finfo(got.dtype).eps / 2
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 2.0 ** -126
    assert got.shape == want.shape and torch.isfinite(got).all(), name
    if got.numel():
        times = float(((got.double() - want).abs() / (terms * UNIT * large + half * (want.abs() + terms * UNIT * large) + tiny)).max())
        assert times <= 1.0, f"{name}: {times} times the bound"


def make(dtype, lead, channels, width, bias=True, state=None, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    x = rand(*lead, channels + 5)[..., 3:channels + 3]
    return x, rand(channels, width), rand(channels) if bias else None, rand(state, width - 1, channels) if state else None


CASES = [(torch.float32, (1, 1), 1, 4), (torch.bfloat16, (3, 2), 24, 4), (torch.float16, (2, 3), 37, 3), (torch.float32, (2, 50), 130, 2), (torch.bfloat16, (1, 700), 520, 4),
         (torch.float16, (4, 33), 64, 4), (torch.float32, (130, 3), 9, 4), (torch.bfloat16, (2, 65), 1001, 3)]


@pytest.mark.parametrize("dtype,lead,channels,width", CASES, ids=str)
@pytest.mark.parametrize("act", ["silu", None], ids=str)
@pytest.mark.parametrize("whole", [True, False], ids=["whole", "bare"])
def test_prompts_and_gradients(tcr, dtype, lead, channels, width, act, whole):
    x, w, bias, state = make(dtype, lead, channels, width, whole, lead[0] if whole else None)
    out, last = tcr.causal_conv(x, w, bias=bias, activation=act, state=state, final_state=True)
    want, large = (reference(x, w, bias, act, None, state, large=m) for m in (False, True))
    check(out, want[0], large[0], 32, "out")
    assert torch.equal(last.double(), want[1])
    dout = torch.randn(*lead, channels + 1, device="cuda").to(dtype)[..., 1:]
    dfinal = torch.randn(lead[0], width - 1, channels, device="cuda").to(dtype) if whole else None
    got = dict(zip(("dx", "dweight", "dbias", "dstate"), tcr.causal_conv_backward(dout, x, w, bias=bias, activation=act, state=state, dfinal=dfinal)))
    assert [k for k in got if got[k] is None] == ([] if whole else ["dbias", "dstate"])
    want, large = (reference(x, w, bias, act, None, state, dout, dfinal, large=m) for m in (False, True))
    for name, g in got.items():
        if g is not None:
            check(g, want[name], large[name], 40 + (lead[0] * lead[1] if name in ("dweight", "dbias") else 0), name)


@pytest.mark.parametrize("dtype,channels,width", [(torch.float32, 70, 4), (torch.bfloat16, 64, 3), (torch.float16, 1033, 4), (torch.float32, 3, 2)], ids=str)
@pytest.mark.parametrize("given", [True, False], ids=["state", "none"])
def test_packed_and_gradients(tcr, dtype, channels, width, given):
    x, w, bias, state = make(dtype, (311,), channels, width, True, 10 if given else None, seed=1)
    outside = torch.ones(311, dtype=torch.bool, device="cuda")
    outside[3:300] = False
    x[outside] = float("nan")
    offsets = torch.tensor(GAPS, device="cuda")
    out, last = tcr.causal_conv(x, w, bias=bias, offsets=offsets, state=state, final_state=True)
    want, large = (reference(x, w, bias, True, offsets, state, large=m) for m in (False, True))
    assert (out[outside] == 0).all()
    check(out, want[0], large[0], 32, "out")
    assert torch.equal(last.double(), want[1])
    dout = torch.randn(311, channels, device="cuda").to(dtype)
    dout[outside] = float("nan")
    dfinal = torch.randn(10, width - 1, channels, device="cuda").to(dtype) if given else None
    got = dict(zip(("dx", "dweight", "dbias", "dstate"), tcr.causal_conv_backward(dout, x, w, bias=bias, offsets=offsets, state=state, dfinal=dfinal)))
    assert (got["dx"][outside] == 0).all()
    want, large = (reference(x, w, bias, True, offsets, state, dout, dfinal, large=m) for m in (False, True))
    for name, g in got.items():
        if g is not None:
            check(g, want[name], large[name], 40 + (297 if name in ("dweight", "dbias") else 0), name)


def test_gradients_against_differences(tcr):
    """Central differences of the definition in 64 bits along a random direction: h = 2^-13, so h^2 / 6 of a third derivative of the loss's own order, 2^-28."""
    x, w, bias, state = make(torch.float32, (2, 40), 12, 4, True, 2, seed=2)
    dout, dfinal = torch.randn(2, 40, 12, device="cuda"), torch.randn(2, 3, 12, device="cuda")
    got = tcr.causal_conv_backward(dout, x, w, bias=bias, state=state, dfinal=dfinal)
    way = [torch.randn_like(t).double() for t in (x, w, bias, state)]

    def loss(step):
        a, b, c, d = (t.double() + step * v for t, v in zip((x, w, bias, state), way))
        out, last = reference(a, b, c, True, None, d)
        return float((out * dout.double()).sum() + (last * dfinal.double()).sum())

    h = 2.0 ** -13
    terms = [(g.double() * v) for g, v in zip(got, way)]
    assert abs((loss(h) - loss(-h)) / (2 * h) - sum(float(t.sum()) for t in terms)) <= 1e-4 * sum(float((t * t).sum()) for t in terms) ** 0.5


@pytest.mark.parametrize("empty", [(0, 5), (3, 0)], ids=str)
def test_nothing(tcr, empty):
    x, w, bias, state = make(torch.float16, empty, 24, 4, True, empty[0])
    out, last = tcr.causal_conv(x, w, bias=bias, state=state, final_state=True)
    assert out.shape == (*empty, 24) and (state is None or torch.equal(last, state))
    dx, dw, db, ds = tcr.causal_conv_backward(torch.zeros_like(out), x, w, bias=bias, state=state, dfinal=state)
    assert (dw == 0).all() and (db == 0).all() and (state is None or torch.equal(ds, state))


@pytest.mark.parametrize("dtype,channels,width", [(torch.float32, 70, 4), (torch.bfloat16, 64, 3), (torch.float16, 1033, 4), (torch.bfloat16, 1, 2)], ids=str)
def test_step_goes_on_like_the_prompt(tcr, dtype, channels, width):
    x, w, bias, state = make(dtype, (5, 7), channels, width, True, 5, seed=3)
    want, end = tcr.causal_conv(x, w, bias=bias, state=state, final_state=True)
    for t in range(7):
        other = torch.empty_like(state)
        got = tcr.causal_conv_step(x[:, t], w, state, bias=bias, new_state=other)
        same = tcr.causal_conv_step(x[:, t], w, state, bias=bias)
        assert torch.equal(state, other) and torch.equal(got, same) and torch.equal(got, want[:, t])
    assert torch.equal(state, end)


def test_infinities_stay_within_reach(tcr):
    x, w, bias, _ = make(torch.float32, (60,), 20, 4, True, None, seed=4)
    offsets = torch.tensor([0, 20, 40, 60], device="cuda")
    clean = tcr.causal_conv(x, w, bias=bias, offsets=offsets)
    x[38, 3], x[10, 5] = float("nan"), float("nan")
    out = tcr.causal_conv(x, w, bias=bias, offsets=offsets)
    hit = torch.zeros(60, 20, dtype=torch.bool, device="cuda")
    hit[38:40, 3], hit[10:14, 5] = True, True
    assert torch.equal(out[~hit], clean[~hit]) and torch.isnan(out[hit]).all()


def test_same_from_run_to_run_and_given_outputs(tcr):
    x, w, bias, state = make(torch.bfloat16, (3, 300), 200, 4, True, 3, seed=5)
    first = tcr.causal_conv_backward(x, x, w, bias=bias, state=state)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, tcr.causal_conv_backward(x, x, w, bias=bias, state=state)))
    wide = torch.full((3, 300, 204), 7.0, device="cuda", dtype=torch.bfloat16)
    got = tcr.causal_conv(x, w, bias=bias, state=state, out=wide[..., 1:201])
    assert torch.equal(got, tcr.causal_conv(x, w, bias=bias, state=state)) and (wide[..., :1] == 7).all() and (wide[..., 201:] == 7).all()


def test_refusals(tcr):
    x, w, bias, state = make(torch.bfloat16, (2, 8), 16, 4, True, 2)
    for bad in ((x.float(), w), (x.cpu(), w), (x, w[:8]), (x, w[:, :1]), (x, w.T.contiguous().T), (x[0], w), (x.transpose(0, 2).contiguous().transpose(0, 2), w)):
        with pytest.raises((TypeError, ValueError)):
            tcr.causal_conv(*bad)
    for more in ({"bias": bias.float()}, {"activation": "relu"}, {"state": state[:1]}, {"state": state.float()}, {"out": x.float()}, {"offsets": torch.tensor([0, 8], device="cuda")}):
        with pytest.raises((TypeError, ValueError)):
            tcr.causal_conv(x, w, **more)
    with pytest.raises(tcr.TcrError):
        tcr.causal_conv(x, torch.zeros(16, 5, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(tcr.TcrError):
        tcr.causal_conv(x, w, out=x)
    with pytest.raises(TypeError):
        tcr.causal_conv_step(x[:, 0], w, state[:, :2])

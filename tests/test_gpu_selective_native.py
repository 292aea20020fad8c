"""The convolution, the selective scan and the clipping through the extension module and through ctypes: the same results, types and errors; what is no plain GPU tensor is
left to binding.py."""
import pytest
import torch

from paper_1811_09736_amd import binding as tcr


def flat(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


def bits(x):
    return x.contiguous().reshape(-1).view(torch.int32 if x.element_size() == 4 else torch.int16)


def same(a, b):
    """Bit for bit: random steps without a softplus are negative too, and a state that grows by exp(2.5) a token leaves the range within 37 tokens: NaN on both sides."""
    a, b = flat(a), flat(b)
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and not x.requires_grad
        assert torch.equal(bits(x), bits(y))


def test_what_is_no_gpu_tensor_is_left_to_binding():
    x, n = torch.zeros(2, 8, 16), tcr._native
    assert n.causal_conv(x, torch.zeros(16, 4), None, "silu", None, None, None, False) is None
    assert n.selective_scan(x, x, torch.zeros(16, 4), torch.zeros(2, 8, 1, 4), torch.zeros(2, 8, 1, 4), None, None, None, True, None, None, None, False) is None
    assert n.gradient_norm([x]) is None and n.clip_gradients([x], 1.0, 1e-6, None) is None and n.gradient_norm([]) is None and n.gradient_norm(3) is None
    with pytest.raises(TypeError, match="x must be"):
        tcr.causal_conv(x, torch.zeros(16, 4))
    with pytest.raises(TypeError, match="x must be"):
        tcr.selective_scan(x, x, torch.zeros(16, 4), torch.zeros(2, 8, 1, 4), torch.zeros(2, 8, 1, 4))
    with pytest.raises(TypeError, match="tensors must be"):
        tcr.clip_gradients([x], 1.0)


@pytest.fixture(scope="module")
def here():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.cuda.current_stream()


def made(*shape, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda").to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32], ids=str)
def test_convolution_both_ways(here, dtype):
    x, w, bias, s = made(2, 40, 70, dtype=dtype)[..., 3:67], made(64, 4, dtype=dtype), made(64, dtype=dtype), made(2, 3, 64, dtype=dtype)
    o, d = torch.tensor([0, 3, 40], device="cuda"), made(2, 40, 64, dtype=dtype)
    for a, more in ((x, {}), (x, {"bias": bias, "activation": None, "state": s, "final_state": True}), (x[0], {"bias": bias, "offsets": o, "state": s, "final_state": True})):
        native = tcr._native.causal_conv(a, w, more.get("bias"), more.get("activation", "silu"), more.get("offsets"), None, more.get("state"), more.get("final_state", False))
        assert native is not None
        same(native, tcr.causal_conv(a, w, stream=here, **more))
        out = torch.empty(a.shape, dtype=dtype, device="cuda")
        got = flat(tcr.causal_conv(a, w, out=out, **more))
        assert got[0] is out
        same(tuple(got), native)
    native = tcr._native.causal_conv_backward(x, w, bias, "silu", None, d, s, s)
    assert native is not None
    same(native, tcr.causal_conv_backward(d, x, w, bias=bias, state=s, dfinal=s, stream=here))
    n1, n2, n3 = torch.empty_like(s), torch.empty_like(s), s.clone()
    native = tcr._native.causal_conv_step(x[:, 0], w, bias, "silu", None, None, s, n1)
    assert native is not None
    same((native, n1), (tcr.causal_conv_step(x[:, 0], w, s, bias, new_state=n2, stream=here), n2))
    same((native, n1), (tcr.causal_conv_step(x[:, 0], w, n3, bias), n3))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32], ids=str)
def test_scan_both_ways(here, dtype):
    x, dt, z = (made(2, 40, 70, dtype=dtype)[..., 3:67] for _ in range(3))
    a, b, c = -torch.rand(64, 16, device="cuda"), made(2, 40, 2, 16, dtype=dtype), made(2, 40, 2, 16, dtype=dtype)
    skip, bias, s = made(64, dtype=torch.float32), made(64, dtype=torch.float32), made(2, 64, 16, dtype=torch.float32)
    o, d = torch.tensor([0, 3, 40], device="cuda"), made(2, 40, 64, dtype=dtype)
    whole = {"skip": skip, "gate": z, "dt_bias": bias, "state": s, "final_state": True}
    for args, more in (((x, dt, a, b, c), {}), ((x, dt, a, b, c), whole), ((x[0], dt[0], a, b[0], c[0]), {**whole, "gate": z[0], "offsets": o, "softplus": False})):
        native = tcr._native.selective_scan(*args, more.get("skip"), more.get("gate"), more.get("dt_bias"), more.get("softplus", True), more.get("offsets"), None,
                                            more.get("state"), more.get("final_state", False))
        assert native is not None
        same(native, tcr.selective_scan(*args, stream=here, **more))
        out = torch.empty(args[0].shape, dtype=dtype, device="cuda")
        got = flat(tcr.selective_scan(*args, out=out, **more))
        assert got[0] is out
        same(tuple(got), native)
    for given, native in (({}, (None, None, None, True, None, d, None, None)), ({"skip": skip, "gate": z, "dt_bias": bias, "state": s, "dfinal": s}, (skip, z, bias, True, None, d, s, s))):
        got = tcr._native.selective_scan_backward(x, dt, a, b, c, *native)
        assert got is not None
        same(got, tcr.selective_scan_backward(d, x, dt, a, b, c, stream=here, **given))
    now = [t[:, 0] if t.dim() > 2 else t for t in (x, dt, a, b, c)]
    n1, n2, n3 = torch.empty_like(s), torch.empty_like(s), s.clone()
    native = tcr._native.selective_scan_step(*now, skip, z[:, 0], bias, True, None, None, s, n1)
    assert native is not None
    given = {"skip": skip, "gate": z[:, 0], "dt_bias": bias}
    same((native, n1), (tcr.selective_scan_step(*now, s, new_state=n2, stream=here, **given), n2))
    same((native, n1), (tcr.selective_scan_step(*now, n3, **given), n3))


@pytest.mark.gpu
def test_clipping_both_ways(here):
    tensors = [made(70, 33), made(5, dtype=torch.float32), made(1000, dtype=torch.float16)]
    same(tcr._native.gradient_norm(tensors), tcr.gradient_norm(tensors, stream=here))
    one, two = ([torch.empty_like(t) for t in tensors] for _ in range(2))
    native = tcr._native.clip_gradients(tensors, 1.0, 1e-6, one)
    assert native is not None and native.dim() == 0
    same((native, *one), (tcr.clip_gradients(tensors, 1.0, out=two, stream=here), *two))
    same(tcr.clip_gradients(iter(tensors), 1), native)                        # what the module leaves: any iterable, whole numbers
    same(tuple(tensors), tuple(one))
    with pytest.raises(tcr.TcrError):
        tcr.clip_gradients([tensors[0], tensors[0]], 1.0)

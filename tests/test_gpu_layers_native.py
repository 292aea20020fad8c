"""Linear attention and the root-mean-square norm through the extension module and through ctypes: the same results, types and errors."""
import pytest
import torch

from paper_1811_09736_amd import binding as tcr


def flat(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


def same(a, b):
    a, b = flat(a), flat(b)
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert x.dtype == y.dtype and x.shape == y.shape and x.device == y.device and not x.requires_grad
        assert torch.equal(x.view(torch.uint8) if x.element_size() == 1 else x, y.view(torch.uint8) if y.element_size() == 1 else y)


@pytest.fixture(scope="module")
def here():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.cuda.current_stream()


def made(*shape, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda").to(dtype)


@pytest.mark.gpu
def test_attention_both_ways(here):
    q, k, v, decay = made(2, 40, 4, 64), made(2, 40, 2, 64), made(2, 40, 2, 48), -torch.rand(4, device="cuda")
    s, d = made(2, 4, 64, 48, dtype=torch.float32), made(2, 40, 4, 48)
    o = torch.tensor([0, 3, 40], device="cuda")
    turned = q.transpose(1, 2).contiguous().transpose(1, 2)
    for a, more in (((q, k, v), {}), ((q, k, v), {"scale": 0.5, "state": s, "final_state": True}), ((turned, k, v), {"final_state": True}),
                    ((q[0], k[0], v[0]), {"offsets": o, "state": s, "final_state": True})):
        native = tcr._native.linear_attention(*a, decay, more.get("scale"), more.get("offsets"), more.get("state"), more.get("final_state", False), None)
        assert native is not None
        same(native, tcr.linear_attention(*a, decay, stream=here, **more))
        same(native, tcr.linear_attention(*a, decay, **more))
        out = torch.empty(*a[0].shape[:-1], 48, dtype=q.dtype, device="cuda")
        got = flat(tcr.linear_attention(*a, decay, out=out, **more))
        assert got[0] is out
        same(tuple(got), native)
    for state, final in ((None, None), (s, s * 2)):
        native = tcr._native.linear_attention_backward(q, k, v, decay, None, None, state, final, d)
        assert native is not None
        same(native, tcr.linear_attention_backward(d, q, k, v, decay, state=state, dfinal=final, stream=here))
    a = (q[:, 0], k[:, 0], v[:, 0])
    n1, n2, n3 = torch.empty_like(s), torch.empty_like(s), s.clone()
    native = tcr._native.linear_attention_step(*a, decay, None, None, s, n1, None)
    same((native, n1), (tcr.linear_attention_step(*a, decay, s, new_state=n2, stream=here), n2))
    same((native, n1), (tcr.linear_attention_step(*a, decay, n3), n3))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_norm_both_ways(here, dtype):
    x, r, w = made(3, 5, 200, dtype=dtype), made(3, 5, 200, dtype=dtype), made(200, dtype=dtype)
    for weight in (w, w.float()):
        for res in (None, r):
            for rstd in (False, True):
                native = tcr._native.rms_norm(x, weight, res, 1e-5, rstd)
                assert native is not None
                same(native, tcr.rms_norm(x, weight, residual=res, eps=1e-5, rstd=rstd, stream=here))
            for kind in (torch.int8, torch.float8_e4m3fn):
                native = tcr._native.rms_norm_quantized(x, weight, res, 1e-5, kind is torch.int8, 64)
                assert native is not None
                same(native, tcr.rms_norm_quantized(x, weight, residual=res, eps=1e-5, dtype=kind, group=64, stream=here))
            root = torch.rand(3, 5, device="cuda")
            native = tcr._native.rms_norm_backward(x, r, weight, root, res)
            assert native is not None
            same(native, tcr.rms_norm_backward(x, r, weight, root, dtotal=res, stream=here))


@pytest.mark.gpu
def test_errors_both_ways(here):
    q, decay = made(1, 10, 2, 64), torch.zeros(2, device="cuda")
    for more in ({}, {"stream": here}):
        with pytest.raises(tcr.TcrError) as e:
            tcr.linear_attention(q[..., :12].contiguous(), q[..., :12].contiguous(), q, decay, **more)
        assert e.value.status == tcr.ERR_UNSUPPORTED
        with pytest.raises(tcr.TcrError) as e:
            tcr.linear_attention(q, q, q, decay, scale=0.0, **more)
        assert e.value.status == tcr.ERR_INVALID_ARG
        with pytest.raises(ValueError):
            tcr.linear_attention(q, q[:, :5], q, decay, **more)
        with pytest.raises(TypeError):
            tcr.linear_attention(q, q, q, decay[:1], **more)
        with pytest.raises(tcr.TcrError):
            tcr.rms_norm(q, q[0, 0, 0].contiguous(), eps=-1.0, **more)


@pytest.mark.parametrize("x", [torch.zeros(2, 8), torch.zeros(2, 8, dtype=torch.float16), [0.0], None], ids=str)
def test_what_is_no_gpu_tensor_is_left_to_binding(x):
    n = tcr._native
    assert n.linear_attention(x, x, x, x, None, None, None, False, None) is None
    assert n.linear_attention_step(x, x, x, x, None, None, x, None, None) is None
    assert n.linear_attention_backward(x, x, x, x, None, None, None, None, x) is None
    assert n.rms_norm(x, x, None, 1e-6, False) is None
    assert n.rms_norm_quantized(x, x, None, 1e-6, False, 0) is None
    assert n.rms_norm_backward(x, x, x, x, None) is None
    if isinstance(x, torch.Tensor):
        with pytest.raises(TypeError):
            tcr.rms_norm(x, x)
        with pytest.raises(TypeError):
            tcr.linear_attention(x[None, None], x[None, None], x[None, None], x[0])

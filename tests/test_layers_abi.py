"""Refusals of linear attention and of the norm that need no GPU: bad shapes, pointers and types come back as a status before any device work."""
import ctypes

import pytest

from paper_1811_09736_amd import binding as tcr

BASE = 1 << 20                               # an aligned address that is never followed


def shape(**more):
    s = dict(dtype=tcr.F16, heads=4, kv_heads=2, dk=64, dv=64, sequences=2, tokens=10, offsets=None, log_decay=BASE, scale=0.125)
    s.update(more)
    a = tcr.AttentionShape()
    for k, v in s.items():
        setattr(a, k, v)
    for n in ("q_stride", "k_stride", "v_stride", "o_stride"):
        getattr(a, n)[:] = [2560, 256, 64]
    return a


def forward(a, q=BASE, k=BASE, v=BASE, out=BASE, state=None, last=None):
    return tcr.raw().tcr_linear_attention(None if a is None else ctypes.byref(a), q, k, v, out, state, last, None)


@pytest.mark.parametrize("more", [{"dtype": tcr.F32}, {"dtype": 9}, {"heads": 0}, {"kv_heads": 0}, {"kv_heads": 3}, {"dk": 0}, {"dv": 0}, {"log_decay": None},
                                  {"log_decay": BASE + 2}, {"offsets": BASE + 4}, {"scale": 0.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"scale": 1e-30}], ids=str)
def test_attention_shapes_that_are_none(more):
    a = shape(**more)
    assert forward(a) == tcr.ERR_INVALID_ARG
    assert tcr.raw().tcr_linear_attention_backward(ctypes.byref(a), *[BASE] * 7, None, None, None, None) == tcr.ERR_INVALID_ARG
    a.tokens = 1
    assert tcr.raw().tcr_linear_attention_step(ctypes.byref(a), *[BASE] * 6, None) == tcr.ERR_INVALID_ARG


@pytest.mark.parametrize("more", [{"dk": 12}, {"dv": 264}, {"dk": 4}, {"tokens": 1 << 31}, {"sequences": 1 << 40}, {"heads": 1 << 17, "kv_heads": 1 << 17},
                                  {"sequences": 1 << 25, "tokens": 1}], ids=str)
def test_attention_sizes_without_a_kernel(more):
    assert forward(shape(**more)) == tcr.ERR_UNSUPPORTED


def test_attention_pointers():
    inv = tcr.ERR_INVALID_ARG
    assert forward(None) == inv
    for name in ("q", "k", "v", "out"):
        assert forward(shape(), **{name: None}) == inv and forward(shape(), **{name: BASE + 1}) == inv
    assert forward(shape(), state=BASE + 4) == inv and forward(shape(), last=BASE + 8) == inv and forward(shape(), state=BASE, last=BASE) == inv
    step = tcr.raw().tcr_linear_attention_step
    assert step(ctypes.byref(shape()), *[BASE] * 6, None) == inv                                     # ten tokens
    assert step(ctypes.byref(shape(tokens=1)), *[BASE] * 4, None, BASE, None) == inv
    assert step(ctypes.byref(shape(tokens=1, offsets=BASE)), *[BASE] * 6, None) == inv
    back = tcr.raw().tcr_linear_attention_backward
    for i in range(7):
        args = [BASE] * 7
        args[i] = None
        assert back(ctypes.byref(shape()), *args, None, None, None, None) == inv
    assert back(ctypes.byref(shape()), *[BASE] * 7, None, BASE, BASE, None) == inv                  # dfinal's place
    # nothing to do
    assert forward(shape(sequences=0), None, None, None, None) == tcr.OK


def test_norm_arguments():
    norm, codes, back = tcr.raw().tcr_rms_norm, tcr.raw().tcr_rms_norm_quantized, tcr.raw().tcr_rms_norm_backward
    inv = tcr.ERR_INVALID_ARG
    assert norm(BASE, None, BASE, BASE, None, None, 4, 0, 8, 8, 1e-6, tcr.F16, tcr.F16, None) == inv
    assert norm(BASE, None, BASE, BASE, None, None, 4, 8, 8, 8, float("nan"), tcr.F16, tcr.F16, None) == inv
    assert norm(BASE, None, BASE, BASE, None, None, 4, 8, 8, 8, 1e-6, tcr.F16, tcr.BF16, None) == inv
    assert norm(BASE, None, BASE, BASE, None, None, 4, 8, 8, 8, 1e-6, tcr.E4M3, tcr.E4M3, None) == inv
    assert norm(BASE + 2, None, BASE, BASE, None, None, 4, 8, 8, 8, 1e-6, tcr.F32, tcr.F32, None) == inv
    assert norm(BASE, BASE + 1, BASE, BASE, None, None, 4, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, None) == inv
    assert norm(BASE, None, BASE, BASE, None, BASE + 2, 4, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, None) == inv
    assert norm(BASE, None, BASE, BASE, None, None, 1 << 31, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, None) == tcr.ERR_UNSUPPORTED
    assert norm(None, None, None, None, None, None, 0, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, None) == tcr.OK
    assert codes(BASE, None, BASE, BASE, None, None, 4, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, tcr.E4M3, 0, None) == inv
    assert codes(BASE, None, BASE, BASE, BASE, None, 4, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, tcr.F16, 0, None) == inv
    assert codes(BASE, None, BASE, BASE, BASE, None, 4, 8, 8, 8, 1e-6, tcr.F16, tcr.F16, tcr.I8, 16, None) == tcr.ERR_UNSUPPORTED
    assert back(BASE, BASE, BASE, BASE, None, BASE, None, 4, 8, 8, 8, 8, tcr.F16, tcr.F16, None) == inv
    assert back(BASE, BASE, BASE, None, None, BASE, BASE, 4, 8, 8, 8, 8, tcr.F16, tcr.F16, None) == inv
    assert back(BASE, BASE, BASE, BASE, BASE + 1, BASE, BASE, 4, 8, 8, 8, 8, tcr.F16, tcr.F16, None) == inv
    assert back(BASE, BASE, BASE, BASE, None, BASE, BASE, 4, 1 << 25, 8, 8, 8, tcr.F16, tcr.F16, None) == tcr.ERR_UNSUPPORTED

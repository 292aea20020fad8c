"""Outputs of linear attention that share memory with what other workgroups still read are refused, which needs no GPU: in front of any device work."""
import ctypes

import pytest

from paper_1811_09736_amd import binding as tcr

BASE = 1 << 30                               # addresses that are never followed
FAR = 1 << 24
H, T, D = 4, 10, 64
ROWS = 2 * 2 * T * H * D                     # bytes of q and of out (k, v: half of them)


def shape(**more):
    a = tcr.AttentionShape()
    for k, v in dict(dtype=tcr.F16, heads=H, kv_heads=H // 2, dk=D, dv=D, sequences=2, tokens=T, offsets=None, log_decay=BASE + 64 * FAR, scale=0.125, **more).items():
        setattr(a, k, v)
    a.q_stride[:] = a.o_stride[:] = [T * H * D, H * D, D]
    a.k_stride[:] = a.v_stride[:] = [T * H * D // 2, H * D // 2, D]
    return a


def forward(a, out, q=BASE, k=BASE + FAR, v=BASE + 2 * FAR, state=None, last=None):
    return tcr.raw().tcr_linear_attention(ctypes.byref(a), q, k, v, out, state, last, None)


@pytest.mark.parametrize("out", [BASE, BASE + FAR, BASE + 2 * FAR, BASE + 2, BASE + ROWS - 2, BASE - ROWS + 2, BASE + FAR + ROWS // 2 - 2, BASE + 2 * FAR - ROWS + 2])
def test_outputs_in_the_inputs_place(out):
    assert forward(shape(), out) == tcr.ERR_INVALID_ARG
    packed = shape()
    packed.offsets, packed.tokens, packed.sequences = BASE + 65 * FAR, 2 * T, 3
    assert forward(packed, out) == tcr.ERR_INVALID_ARG


def test_a_steps_output():
    a = shape()
    a.tokens = 1
    a.sequences = 20
    a.q_stride[:] = a.o_stride[:] = [H * D, 0, D]
    a.k_stride[:] = a.v_stride[:] = [H * D // 2, 0, D]
    step = tcr.raw().tcr_linear_attention_step
    for out in (BASE, BASE + FAR, BASE + 2 * FAR, BASE + 2, BASE + ROWS - 2):
        assert step(ctypes.byref(a), BASE, BASE + FAR, BASE + 2 * FAR, out, BASE + 3 * FAR, BASE + 3 * FAR, None) == tcr.ERR_INVALID_ARG


def test_rows_with_gaps_that_start_where_others_do():
    a = shape()
    a.o_stride[:] = [T * H * D * 2, H * D * 2, D]
    for out in (BASE, BASE + FAR, BASE + 2 * FAR):
        assert forward(a, out) == tcr.ERR_INVALID_ARG


def test_states_that_overlap():
    out, state = BASE + 10 * FAR, BASE + 20 * FAR
    size = 4 * 2 * H * D * D
    for last in (state, state + 16, state + size - 16, state - size + 16):
        assert forward(shape(), out, state=state, last=last) == tcr.ERR_INVALID_ARG
    a = shape()
    a.tokens = 1
    step = tcr.raw().tcr_linear_attention_step
    for new in (state + 16, state + size - 16, state - size + 16):
        assert step(ctypes.byref(a), BASE, BASE + FAR, BASE + 2 * FAR, out, state, new, None) == tcr.ERR_INVALID_ARG
    back = tcr.raw().tcr_linear_attention_backward
    ins = [BASE + i * FAR for i in range(7)]
    for dstate in (state, state + 16, state - size + 16):
        assert back(ctypes.byref(shape()), *ins, None, state, dstate, None) == tcr.ERR_INVALID_ARG

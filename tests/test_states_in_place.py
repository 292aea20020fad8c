"""States that stand in the place of what the same call writes or reads are refused (no GPU: it comes back before any device work)."""
import ctypes

import pytest

from paper_1811_09736_amd import binding as tcr
from test_selective_abi import BASE, FAR, conv, forward, scan, selective

INV = tcr.ERR_INVALID_ARG
OUT = 2 * 10 * 64 * 2                            # bytes of out: 2 sequences, 10 tokens, 64 channels of 16 bits


@pytest.mark.parametrize("at", [FAR, FAR + 128, FAR + OUT - 4, FAR - 64], ids=["same", "inside", "end", "front"])
def test_states_on_outputs(at):
    """2 x 3 x 64 elements of 16 bits of the convolution, 2 x 64 x 16 floats of the scan."""
    assert forward(conv(), last=at) == INV and forward(conv(), state=at) == INV
    assert selective(scan(), last=at) == INV and selective(scan(), state=at) == INV


def test_last_states_on_inputs():
    assert forward(conv(), last=BASE) == INV and forward(conv(), last=BASE + 128) == INV
    far = FAR * 4
    for name in ("x", "dt", "b", "c", "gate"):
        assert selective(scan(), **{name: far, "last": far}) == INV and selective(scan(), **{name: far, "last": far + 64}) == INV


def test_steps():
    wide = [64, 0]
    one = conv(tokens=1, x_stride=wide, o_stride=wide)
    for state, new in ((FAR, FAR * 2), (FAR * 2, FAR), (FAR, FAR), (FAR + 64, FAR + 64)):
        assert tcr.raw().tcr_causal_conv_step(ctypes.byref(one), BASE, BASE, None, FAR, state, new, None) == INV
        one_scan = scan(tokens=1, x_stride=wide, dt_stride=wide, gate_stride=wide, o_stride=wide, b_stride=[16, 0, 16], c_stride=[16, 0, 16])
        assert tcr.raw().tcr_selective_scan_step(ctypes.byref(one_scan), *[BASE] * 4, None, FAR, state, new, None) == INV

"""Which rows of an output share elements: the check on the host against counting, and what the calls refuse (no GPU: it comes back before any device work)."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_1811_09736_amd import binding as tcr
from test_selective_abi import conv, forward, scan, selective

LAYERS = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1811_09736_amd", "csrc", "layers")

COUNTING = r"""
#include <cstdio>
#include <set>
#include "tcr_lattice.hpp"
static bool counted(uint64_t n0, int64_t s0, uint64_t n1, int64_t s1, uint64_t wide) {
    std::set<int64_t> seen;
    for (uint64_t i = 0; i < n0; ++i)
        for (uint64_t j = 0; j < n1; ++j)
            for (uint64_t k = 0; k < wide; ++k)
                if (!seen.insert((int64_t)i * s0 + (int64_t)j * s1 + (int64_t)k).second) return true;
    return false;
}
int main() {
    long calls = 0, meeting = 0;
    const uint64_t counts[] = {0, 1, 2, 3, 5, 8, 13};
    for (uint64_t n0 : counts)
        for (uint64_t n1 : counts)
            for (int64_t s0 = -20; s0 <= 44; ++s0)
                for (int64_t s1 = -13; s1 <= 40; ++s1)
                    for (uint64_t wide : {1, 2, 3, 5, 8}) {
                        const bool want = counted(n0, s0, n1, s1, wide);
                        if (tcr::layers::lattice_meets(n0, s0, n1, s1, wide) != want) {
                            std::printf("%d x %d, %d x %d, %d: %d\n", (int)n0, (int)s0, (int)n1, (int)s1, (int)wide, (int)want);
                            return 1;
                        }
                        ++calls;
                        meeting += want;
                    }
    // long ones: steps of p and q without a common divisor meet from (q, 0) = (0, p) on, not earlier
    const int64_t p = 1000003, q = 999983;
    using tcr::layers::lattice_meets;
    if (lattice_meets(q, p, p, q, 1) || !lattice_meets(q + 1, p, p + 1, q, 1) || lattice_meets(1ull << 40, 7, 7, 1, 1) || !lattice_meets(1ull << 40, 7, 8, 1, 1)) return 2;
    if (!lattice_meets(1ull << 30, INT64_MIN, 1ull << 30, INT64_MIN, 64) || lattice_meets(2, INT64_MIN, 2, INT64_MAX, 1)) return 3;
    std::printf("%ld %ld\n", calls, meeting);
    return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_against_counting(tmp_path):
    source, exe = tmp_path / "lattice.cpp", str(tmp_path / "lattice")
    source.write_text(COUNTING)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", LAYERS, "-o", exe, str(source)], check=True)
    got = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert got.returncode == 0, got.stdout
    calls, meeting = map(int, got.stdout.split())
    assert calls == 7 * 7 * 65 * 54 * 5 and 0 < meeting < calls


@pytest.mark.parametrize("stride", [[64, 64], [128, 64], [576, 64], [600, 64], [100, 128], [127, 100], [-64, 64], [250, 200], [64, 64 * 2 - 1]], ids=str)
def test_rows_of_two_sequences_in_the_same_place(stride):
    """2 sequences of 10 tokens, 64 channels: every step is at least a row, and a row of the second sequence stands on one of the first."""
    assert forward(conv(o_stride=stride)) == tcr.ERR_INVALID_ARG
    assert selective(scan(o_stride=stride)) == tcr.ERR_INVALID_ARG


def test_of_many_sequences():
    assert forward(conv(sequences=1 << 14, tokens=1 << 10, o_stride=[64 * 3, 64 * (1 << 10)])) == tcr.ERR_INVALID_ARG      # token 3 of sequence 0 is token 0 of sequence 1024
    assert tcr.raw().tcr_selective_scan(ctypes.byref(scan(sequences=3, tokens=1000, o_stride=[64 * 7, 64 * 2])), *[1 << 20] * 4, None, 1 << 30, None, None, None) == tcr.ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("shape,stride", [((2, 3), (300, 200)), ((3, 5), (64, 192)), ((7, 4), (65, 7 * 65)), ((2, 10), (640, 64)), ((1, 10), (0, 64)), ((10, 1), (64, 0)), ((2, 5), (100, 200))],
                         ids=str)
def test_rows_between_each_other_are_taken(shape, stride):
    """Rows that lie between those of other sequences without sharing anything: the same values as in an array of their own, and nothing beside them."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    x, taps = torch.randn(*shape, 64, device="cuda"), torch.randn(64, 4, device="cuda")
    a, b = -torch.rand(64, 16, device="cuda"), torch.randn(*shape, 1, 16, device="cuda")
    for call in (lambda **k: tcr.causal_conv(x, taps, **k), lambda **k: tcr.selective_scan(x, x, a, b, b, **k)):
        room = torch.full((4096,), 7.0, device="cuda")
        out = room.as_strided((*shape, 64), (*stride, 1))
        want = call()
        assert torch.equal(call(out=out), want)
        out.fill_(7.0)
        assert (room == 7.0).all()

"""The workspace of linear attention's and the norm's gradients: refusals come before any work, a recorded call that lacks room records nothing, and states between
blocks take no more than the header says."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


class Backward:
    """tcr_linear_attention_backward of `tokens` tokens with shared heads, on given outputs."""

    def __init__(self, tcr, tokens=3000, heads=4, kv=2, d=64):
        self.tcr = tcr
        make = lambda h: torch.randn(1, tokens, h, d, device="cuda").bfloat16()  # noqa: E731
        self.q, self.k, self.v, self.dout = make(heads), make(kv), make(kv), make(heads)
        self.decay = torch.full((heads,), -0.01, device="cuda")
        self.out = [torch.full_like(x, 7.0) for x in (self.q, self.k, self.v)]
        a = self.shape = tcr.AttentionShape()
        a.dtype, a.heads, a.kv_heads, a.dk, a.dv, a.sequences, a.tokens, a.scale = tcr.BF16, heads, kv, d, d, 1, tokens, 0.125
        a.offsets, a.log_decay = None, self.decay.data_ptr()
        a.q_stride[:] = a.o_stride[:] = [tokens * heads * d, heads * d, d]
        a.k_stride[:] = a.v_stride[:] = [tokens * kv * d, kv * d, d]
        # as the header has it: the heads' own gradients in binary32, in the second half of what follows a buffer's first 256 bytes
        self.bytes = 256 + 2 * 4 * tokens * heads * d

    def call(self, stream):
        ins = [x.data_ptr() for x in (self.dout, self.q, self.k, self.v, *self.out)]
        return self.tcr.raw().tcr_linear_attention_backward(ctypes.byref(self.shape), *ins, None, None, None, stream.cuda_stream)

    def untouched(self):
        torch.cuda.synchronize()
        return all((x == 7).all().item() for x in self.out)


def test_a_refused_call_has_done_nothing(tcr):
    b = Backward(tcr)
    for size in (1 << 12, b.bytes - 512):
        tcr.set_workspace(torch.empty(size, dtype=torch.uint8, device="cuda"))
        try:
            assert b.call(torch.cuda.current_stream()) == tcr.ERR_WORKSPACE and b.untouched()
        finally:
            tcr.set_workspace(None)
    tcr.set_workspace(torch.empty(b.bytes, dtype=torch.uint8, device="cuda"))
    try:
        assert b.call(torch.cuda.current_stream()) == tcr.OK and not b.untouched()
    finally:
        tcr.set_workspace(None)
    want = tcr.linear_attention_backward(b.dout, b.q, b.k, b.v, b.decay, scale=0.125)
    for got, w in zip(b.out, want):
        # (fewer blocks: other roundings of sums in 32 bits, then one to bfloat16)
        assert (got.float() - w.float()).norm() <= 2.0 ** -8 * w.float().norm()


def test_recording_without_room_records_nothing(tcr):
    b = Backward(tcr)
    stream = torch.cuda.Stream()                # (one that has no workspace yet)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        marker = torch.zeros(1, device="cuda").add_(1)
        status = b.call(stream)
    assert status == tcr.ERR_UNSUPPORTED
    graph.replay()
    assert b.untouched() and marker.item() == 1
    with torch.cuda.stream(stream):             # outside of the recording it goes, and after that inside too
        assert b.call(stream) == tcr.OK
    torch.cuda.synchronize()
    want = [x.clone() for x in b.out]
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph(), stream=stream):
        status = b.call(stream)
    assert status == tcr.OK
    for _ in range(3):
        for x in b.out:
            x.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(b.out, want))


def test_recording_norm_gradients_without_room(tcr):
    x, w = torch.randn(300, 1000, device="cuda"), torch.ones(1000, device="cuda")
    rstd = torch.rsqrt(x.square().mean(1))
    dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        marker = torch.zeros(1, device="cuda").add_(1)
        status = tcr.raw().tcr_rms_norm_backward(x.data_ptr(), x.data_ptr(), w.data_ptr(), rstd.data_ptr(), None, dx.data_ptr(), dw.data_ptr(), 300, 1000,
                                                 1000, 1000, 1000, tcr.F32, tcr.F32, stream.cuda_stream)
    assert status == tcr.ERR_UNSUPPORTED
    graph.replay()
    torch.cuda.synchronize()
    assert (dx == 7).all() and (dw == 7).all() and marker.item() == 1


@pytest.mark.parametrize("batch,tokens,heads,dk,dv", [(15, 1024, 16, 256, 256), (9, 1024, 16, 256, 256), (3, 4096, 20, 200, 256), (1, 32768, 4, 256, 256),
                                                      (7, 4096, 33, 128, 128), (31, 1024, 8, 128, 128), (5, 3000, 24, 128, 64), (1, 60000, 3, 64, 64)])
def test_states_between_blocks_stay_within_64_mib(tcr, batch, tokens, heads, dk, dv):
    q = torch.zeros(batch, tokens, heads, dk, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros(batch, tokens, heads, dv, device="cuda", dtype=torch.bfloat16)
    decay, out, stream = torch.full((heads,), -0.01, device="cuda"), torch.empty_like(v), torch.cuda.Stream()
    # (the same call once: the stream's queue and the kernels are there before anything is measured, the workspace no longer)
    torch.cuda.synchronize()
    tcr.linear_attention(q, q, v, decay, out=out, stream=stream)
    torch.cuda.synchronize()
    tcr.release_stream(stream)
    before = torch.cuda.mem_get_info()[0]
    tcr.linear_attention(q, q, v, decay, out=out, stream=stream)
    torch.cuda.synchronize()
    taken = before - torch.cuda.mem_get_info()[0]
    tcr.release_stream(stream)
    # (memory is handed out in pieces of 2 MiB)
    assert taken <= (64 << 20) + (2 << 20), taken / 2 ** 20

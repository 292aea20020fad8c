"""Calls that need more threads than one launch may have (2^32): rows of the norm, sequences and heads of linear attention, tokens and elements beside them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


@pytest.fixture(autouse=True)
def free_afterwards():
    yield
    torch.cuda.empty_cache()                 # (tens of GiB that the next test may want to see free)


def parts(n):
    """Slices of the rows to look at: both ends and where a launch of 2^32 threads would end."""
    return [slice(0, 1000), slice(n // 2 - 500, n // 2 + 500), slice(n - 1000, n)]


@pytest.mark.parametrize("rows,cols", [((1 << 29) + 3, 8), ((1 << 28) + 5, 72)])
def test_rows_of_the_norm(tcr, rows, cols):
    # (one row in memory)
    x, w = torch.randn(1, cols, device="cuda").bfloat16(), torch.ones(cols, device="cuda").bfloat16()
    want = tcr.rms_norm(x, w)
    got, rstd = tcr.rms_norm(x.expand(rows, cols), w, rstd=True)
    for part in parts(rows):
        assert (got[part] == want).all() and (rstd[part] == rstd[0]).all()


@pytest.mark.parametrize("rows,cols", [((1 << 25) + 3, 520), ((1 << 22) + 3, 16392)])
def test_rows_of_several_wavefronts(tcr, rows, cols):
    x, w = torch.randn(1, cols, device="cuda").bfloat16(), torch.ones(cols, device="cuda").bfloat16()
    want, scale = tcr.rms_norm_quantized(x, w, dtype=torch.int8)
    got, scales = tcr.rms_norm_quantized(x.expand(rows, cols), w, dtype=torch.int8)
    for part in parts(rows):
        assert (got[part] == want).all() and (scales[part] == scale).all()


def test_single_tokens_of_many_sequences(tcr):
    batch, heads = (1 << 20) + 1, 16
    q, k, v = (torch.randn(1, heads, 8, device="cuda").half().expand(batch, heads, 8) for _ in range(3))
    decay, state = -torch.rand(heads, device="cuda"), torch.randn(1, heads, 8, 8, device="cuda")
    want_state = state.clone()
    want = tcr.linear_attention_step(q[:1], k[:1], v[:1], decay, want_state)
    states = state.expand(batch, heads, 8, 8).contiguous()
    got = tcr.linear_attention_step(q, k, v, decay, states)
    for part in parts(batch):
        assert (got[part] == want).all() and (states[part] == want_state).all()


def test_chunks_of_many_sequences(tcr):
    batch, heads, tokens = (1 << 20) + 1, 16, 3
    q, k, v = (torch.randn(1, tokens, heads, 8, device="cuda").half().expand(batch, tokens, heads, 8) for _ in range(3))
    decay = -torch.rand(heads, device="cuda")
    # (as many as go the same way: through a chunk)
    want, last = tcr.linear_attention(q[:100], k[:100], v[:100], decay, final_state=True)
    got, states = tcr.linear_attention(q, k, v, decay, final_state=True)
    for part in parts(batch):
        assert (got[part] == want[0]).all() and (states[part] == last[0]).all()


def test_tokens_outside_every_sequence(tcr):
    total = (1 << 30) + 70
    q = torch.ones(1, 1, 8, device="cuda", dtype=torch.half).expand(total, 1, 8)
    out = torch.full((total, 1, 8), 7.0, device="cuda", dtype=torch.half)
    offsets = torch.zeros(1, dtype=torch.int64, device="cuda")
    tcr.linear_attention(q, q, q, torch.zeros(1, device="cuda"), offsets=offsets, out=out)
    for part in parts(total):
        assert (out[part] == 0).all()


def test_gradients_of_many_shared_elements(tcr):
    # 2^32 elements of shared keys, and as many values, each the sum over two heads (every token's rows are the same ones in memory)
    tokens, heads, kv, d = (1 << 20) + 1, 32, 16, 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    q, k, v, dout = (torch.randn(1, 1, h, d, generator=gen, device="cuda").bfloat16() for h in (heads, kv, kv, heads))
    decay = torch.full((heads,), -1.0, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    long = [x.expand(1, tokens, x.shape[2], d) for x in (dout, q, k, v)]
    with torch.cuda.stream(stream):
        dq, dk, dv, _ = tcr.linear_attention_backward(*long, decay, scale=0.0625)
    stream.synchronize()
    del dq
    # behind a token stand `n` more: dk = scale * sum of lambda^i over them and itself * sum over the heads of (dout . v) q
    q, k, v, dout = (x[0, 0].double() for x in (q, k, v, dout))
    k, v = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
    each_k = 0.0625 * (dout * v).sum(1, keepdim=True) * q
    each_v = 0.0625 * (q * k).sum(1, keepdim=True) * dout
    for t in (0, tokens // 2, tokens - 70, tokens - 2, tokens - 1):
        times = (1 - torch.exp(torch.tensor(-float(tokens - t), device="cuda", dtype=torch.float64))) / (1 - torch.exp(torch.tensor(-1.0, device="cuda", dtype=torch.float64)))
        for got, each in ((dk, each_k), (dv, each_v)):
            want, size = (times * x.view(kv, 2, d).sum(1) for x in (each, each.abs()))
            # one rounding to bfloat16, two-part factors of 2^-17 (as the header of the kernels has it) in front of it
            assert ((got[0, t].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * size).all(), t
    tcr.release_stream(stream)

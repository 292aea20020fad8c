"""Linear attention with decay against its definition in 64 bits: prompts, packed prompts, single tokens, gradients.

Tolerances.  Outputs are rounded to their type once (by u = 2^-8 relative for bfloat16, 2^-11 for binary16); the factors of what is summed
for them in binary32 may have roundings of that size (a score, a state as a factor), of terms whose magnitudes add up
to `size`, of either sign: |got - want| <= 2 u size.  (Terms add up to more than their sum, so the bound holds for outputs near 0.)
States are binary32 sums of products kept to 2^-22 at least: |got - want| <= 2^-18 size."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_SPACING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


def make(gen, *shape, dtype=torch.float32, spread=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * spread).to(dtype)


def problem(seed, dtype, batch, tokens, heads, kv, dk, dv, offsets=None, state=True):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lead = (batch, tokens) if offsets is None else (tokens,)
    q, k, v = make(gen, *lead, heads, dk, dtype=dtype), make(gen, *lead, kv, dk, dtype=dtype), make(gen, *lead, kv, dv, dtype=dtype)
    decay = -torch.rand(heads, generator=gen, device="cuda") * torch.tensor([0.3, 0.01, 0.0005], device="cuda").repeat(heads)[:heads]
    count = batch if offsets is None else len(offsets) - 1
    s = make(gen, count, heads, dk, dv, spread=3.0) if state else None
    dout, dfinal = make(gen, *lead, heads, dv, dtype=dtype), make(gen, count, heads, dk, dv)
    o = None if offsets is None else torch.tensor(offsets, dtype=torch.int64, device="cuda")
    return q, k, v, decay, o, s, dout, dfinal


def definition(q, k, v, decay, offsets, s, scale):
    """(out, last, size of out, size of last) of the definition in 64 bits, by the sum over pairs of tokens; differentiable."""
    q, k, v, decay = q.double(), k.double(), v.double(), decay.double()
    heads, group = q.shape[-2], q.shape[-2] // k.shape[-2]
    if offsets is None:
        parts = [(q[b], k[b], v[b]) for b in range(q.shape[0])]
    else:
        cuts = offsets.tolist()
        parts = [(q[a:b], k[a:b], v[a:b]) for a, b in zip(cuts, cuts[1:])]
    outs, lasts, out_sizes, last_sizes = [], [], [], []
    for n, (a, b, c) in enumerate(parts):
        a, b, c = a.transpose(0, 1), b.transpose(0, 1).repeat_interleave(group, 0), c.transpose(0, 1).repeat_interleave(group, 0)
        t = torch.arange(a.shape[1], device=a.device, dtype=torch.float64)
        rel = t[:, None] - t[None, :]
        w = torch.where(rel >= 0, torch.exp(decay[:, None, None] * rel.clamp(min=0)), 0.0)
        pre, to_end = torch.exp(decay[:, None] * (t + 1))[..., None], torch.exp(decay[:, None] * (len(t) - 1 - t))[..., None]
        s0 = torch.zeros(heads, a.shape[2], c.shape[2], dtype=torch.float64, device=a.device) if s is None else s[n].double()
        end = torch.exp(decay * len(t))[:, None, None]
        outs.append((scale * (torch.matmul(torch.matmul(a, b.transpose(1, 2)) * w, c) + pre * torch.matmul(a, s0))).transpose(0, 1))
        lasts.append(torch.matmul((b * to_end).transpose(1, 2), c) + end * s0)
        with torch.no_grad():
            out_sizes.append((abs(scale) * (torch.matmul(torch.matmul(a.abs(), b.abs().transpose(1, 2)) * w, c.abs())
                                            + pre * torch.matmul(a.abs(), s0.abs()))).transpose(0, 1))
            last_sizes.append(torch.matmul((b.abs() * to_end).transpose(1, 2), c.abs()) + end * s0.abs())
    join = torch.stack if offsets is None else torch.cat
    return join(outs), torch.stack(lasts), join(out_sizes), torch.stack(last_sizes)


def near(got, want, size, u):
    assert got.shape == want.shape
    off = (got.double() - want).abs() - (2 * u * size + 1e-30)
    assert not torch.isnan(got).any() and (off <= 0).all(), (off.max().item(), (off > 0).sum().item())


def check(tcr, p, scale=None):
    q, k, v, decay, offsets, s, dout, dfinal = p
    u = HALF_SPACING[q.dtype]
    real = q.shape[-1] ** -0.5 if scale is None else scale
    want, last, size, last_size = definition(q, k, v, decay, offsets, s, real)
    got, got_last = tcr.linear_attention(q, k, v, decay, scale=scale, offsets=offsets, state=s, final_state=True)
    assert got.dtype == q.dtype and got_last.dtype == torch.float32
    near(got, want, size, u)
    near(got_last, last, last_size, 2.0 ** -19)
    if s is None:
        assert torch.equal(tcr.linear_attention(q, k, v, decay, scale=scale, offsets=offsets), got)


def check_gradients(tcr, p, scale=None, dfinal=True):
    q, k, v, decay, offsets, s, dout, df = p
    u = HALF_SPACING[q.dtype]
    real = q.shape[-1] ** -0.5 if scale is None else scale
    ins = [x.double().requires_grad_() for x in (q, k, v)] + ([s.double().requires_grad_()] if s is not None else [])
    out, last, _, _ = definition(*ins[:3], decay, offsets, ins[3] if s is not None else None, real)
    loss = (out * dout.double()).sum() + ((last * df.double()).sum() if dfinal else 0.0)
    want = torch.autograd.grad(loss, ins)
    # the sizes: the same gradients of the magnitudes, whose terms are all positive
    big = [x.double().abs().requires_grad_() for x in (q, k, v)] + ([s.double().abs().requires_grad_()] if s is not None else [])
    out, last, _, _ = definition(*big[:3], decay, offsets, big[3] if s is not None else None, abs(real))
    loss = (out * dout.double().abs()).sum() + ((last * df.double().abs()).sum() if dfinal else 0.0)
    size = torch.autograd.grad(loss, big)
    got = tcr.linear_attention_backward(dout, q, k, v, decay, scale=scale, offsets=offsets, state=s, dfinal=df if dfinal else None)
    for g, w, z in zip(got[:3], want, size):
        assert g.dtype == q.dtype
        near(g, w, z, u)
    if s is None:
        assert got[3] is None
    else:
        near(got[3], want[3], size[3], 2.0 ** -19)


TOKENS = [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 200, 513, 1000]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens", TOKENS)
def test_lengths(tcr, dtype, tokens):
    check(tcr, problem(tokens, dtype, 2, tokens, 3, 3, 64, 64))
    check(tcr, problem(tokens, dtype, 1, tokens, 2, 1, 128, 128, state=False))


@pytest.mark.parametrize("dk,dv", [(8, 8), (16, 40), (40, 16), (64, 128), (128, 64), (72, 136), (256, 256), (256, 8), (8, 256), (192, 200)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_widths(tcr, dtype, dk, dv):
    p = problem(dk + dv, dtype, 1, 150, 2, 2, dk, dv)
    check(tcr, p)
    check_gradients(tcr, p)


@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 1), (6, 2), (8, 8)])
def test_shared_keys_and_values(tcr, heads, kv):
    for dtype in (torch.float16, torch.bfloat16):
        p = problem(heads + kv, dtype, 2, 130, heads, kv, 64, 64)
        check(tcr, p)
        check_gradients(tcr, p)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 200, 513])
def test_gradients(tcr, dtype, tokens):
    check_gradients(tcr, problem(tokens + 7, dtype, 2, tokens, 3, 3, 64, 128))
    check_gradients(tcr, problem(tokens + 9, dtype, 1, tokens, 2, 2, 128, 64, state=False), dfinal=False)


PACKED = [[0, 5], [0, 0, 1, 1, 2, 300], [0, 64, 128, 192], [0, 63, 64, 129, 129, 129, 700], [0, 0, 0], [0, 1, 2, 3, 4, 5, 6, 7, 8, 400, 401],
          [0] + list(range(37, 37 * 40, 37)), [0, 1500, 1501, 3000]]


@pytest.mark.parametrize("cuts", PACKED, ids=lambda c: f"{len(c) - 1}x{c[-1]}")
def test_packed_sequences(tcr, cuts):
    for dtype in (torch.float16, torch.bfloat16):
        p = problem(sum(cuts), dtype, 1, cuts[-1], 4, 2, 64, 64, offsets=cuts)
        check(tcr, p)
        check_gradients(tcr, p)


def test_packed_rows_outside_every_sequence_are_zero(tcr):
    cuts = [70, 100, 100, 300]
    q, k, v, decay, o, s, dout, dfinal = problem(3, torch.bfloat16, 1, 400, 2, 2, 64, 64, offsets=cuts)
    k[300:] = float("nan")
    v[:70] = float("inf")
    got = tcr.linear_attention(q, k, v, decay, offsets=o, state=s)
    want, _, size, _ = definition(q, k, v, decay, o, s, 64 ** -0.5)
    near(got[70:300], want, size, HALF_SPACING[torch.bfloat16])
    assert (got[:70] == 0).all() and (got[300:] == 0).all()
    dq, dk, dv, ds = tcr.linear_attention_backward(dout, q, k, v, decay, offsets=o, state=s)
    for g in (dq, dk, dv):
        assert (g[:70] == 0).all() and (g[300:] == 0).all() and torch.isfinite(g).all()


def test_no_tokens_and_no_sequences(tcr):
    q, k, v, decay, o, s, dout, dfinal = problem(3, torch.float16, 2, 0, 2, 2, 64, 64)
    out, last = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
    assert out.numel() == 0 and torch.equal(last, s)
    assert torch.equal(tcr.linear_attention_backward(dout, q, k, v, decay, state=s, dfinal=dfinal)[3], dfinal)
    q, k, v, decay, o, s, dout, dfinal = problem(3, torch.float16, 0, 5, 2, 2, 64, 64)
    out, last = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
    assert out.numel() == 0 and last.numel() == 0
    q, k, v, decay, o, s, dout, dfinal = problem(3, torch.float16, 1, 0, 2, 2, 64, 64, offsets=[0, 0, 0])
    out, last = tcr.linear_attention(q, k, v, decay, offsets=o, state=s, final_state=True)
    assert torch.equal(last, s)
    out, last = tcr.linear_attention(q, k, v, decay, offsets=o, final_state=True)
    assert (last == 0).all()


@pytest.mark.parametrize("value", [0.0, -1e-6, -40.0, -200.0, float("-inf")])
def test_extreme_decays(tcr, value):
    for tokens in (1, 70, 300):
        q, k, v, decay, o, s, dout, dfinal = problem(tokens, torch.bfloat16, 1, tokens, 2, 2, 64, 64)
        decay = torch.full_like(decay, value)
        if value == float("-inf"):               # (the oracle: nothing of the state is left after one token)
            oracle = torch.full_like(decay, -1e4)
        else:
            oracle = decay
        want, last, size, last_size = definition(q, k, v, oracle, o, s, 0.125)
        got, got_last = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
        near(got, want, size, HALF_SPACING[torch.bfloat16])
        near(got_last, last, last_size, 2.0 ** -19)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("factor", [300.0, 1e-3])
def test_scores_and_states_beyond_binary16(tcr, dtype, factor):
    # scores up to 300^2 * 30 and states beyond that, which binary16 does not hold; and ones that it holds only to a few bits
    for tokens in (40, 300):
        q, k, v, decay, o, s, dout, dfinal = problem(5, dtype, 1, tokens, 2, 2, 64, 64)
        q, k = (q.float() * factor).to(dtype), (k.float() * factor).to(dtype)
        v = (v.float() / (factor if factor > 1 else 1.0)).to(dtype)
        s = s * (factor if factor > 1 else 1e-3)
        scale = 1.0 / (factor if factor > 1 else 1e-3)
        want, last, size, last_size = definition(q, k, v, decay, o, s, scale)
        got, got_last = tcr.linear_attention(q, k, v, decay, scale=scale, state=s, final_state=True)
        near(got, want, size, HALF_SPACING[dtype])
        near(got_last, last, last_size, 2.0 ** -19)


@pytest.mark.parametrize("tokens", [70, 600])
def test_strides_and_alignment(tcr, tokens):
    for dtype in (torch.float16, torch.bfloat16):
        q, k, v, decay, o, s, dout, dfinal = problem(11, dtype, 2, tokens, 4, 2, 64, 64)
        want = tcr.linear_attention(q, k, v, decay, state=s)
        grads = tcr.linear_attention_backward(dout, q, k, v, decay, state=s, dfinal=dfinal)
        # [B, H, T, D] in memory; parts of a wider row; rows on odd elements
        views = []
        for x in (q, k, v, dout):
            turned = x.transpose(1, 2).contiguous().transpose(1, 2)
            wide = torch.empty(*x.shape[:3], x.shape[3] + 24, dtype=dtype, device="cuda")[..., 8:8 + x.shape[3]]
            wide.copy_(x)
            uneven = torch.empty(*x.shape[:3], x.shape[3] + 5, dtype=dtype, device="cuda")[..., 3:3 + x.shape[3]]
            uneven.copy_(x)
            views.append((turned, wide, uneven))
        for i in range(3):
            a, b, c, d = (views[j][(i + j) % 3] for j in range(4))
            assert torch.equal(tcr.linear_attention(a, b, c, decay, state=s), want)
            for g, w in zip(tcr.linear_attention_backward(d, a, b, c, decay, state=s, dfinal=dfinal), grads):
                assert torch.equal(g, w)
            out = torch.empty_like(views[3][i])
            out = torch.empty(2, tokens, 4, 69, dtype=dtype, device="cuda")[..., 1:65] if i == 2 else out
            assert torch.equal(tcr.linear_attention(a, b, c, decay, state=s, out=out), want)


@pytest.mark.parametrize("batch", [1, 3, 70])
@pytest.mark.parametrize("dk,dv,heads,kv", [(64, 64, 4, 4), (128, 128, 4, 2), (24, 72, 3, 1), (256, 256, 2, 2)])
def test_single_tokens(tcr, batch, dk, dv, heads, kv):
    for dtype in (torch.float16, torch.bfloat16):
        q, k, v, decay, o, s, dout, dfinal = problem(batch, dtype, batch, 1, heads, kv, dk, dv)
        want, last, size, last_size = definition(q, k, v, decay, None, s, dk ** -0.5)
        new = torch.empty_like(s)
        before = s.clone()
        got = tcr.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, s, new_state=new)
        near(got, want[:, 0], size[:, 0], HALF_SPACING[dtype])
        near(new, last, last_size, 2.0 ** -21)
        assert torch.equal(s, before)
        assert torch.equal(tcr.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, s), got)
        assert torch.equal(s, new)


def test_steps_go_on_from_a_prompt(tcr):
    q, k, v, decay, o, s, dout, dfinal = problem(21, torch.bfloat16, 2, 140, 4, 2, 128, 128)
    want, last, size, last_size = definition(q, k, v, decay, None, s, 128 ** -0.5)
    out, state = tcr.linear_attention(q[:, :133], k[:, :133], v[:, :133], decay, state=s, final_state=True)
    rows = [out]
    for t in range(133, 140):
        rows.append(tcr.linear_attention_step(q[:, t], k[:, t], v[:, t], decay, state)[:, None])
    near(torch.cat(rows, 1), want, size, HALF_SPACING[torch.bfloat16])
    near(state, last, last_size, 2.0 ** -19)


def test_gradients_by_differences(tcr):
    # the loss along a direction, by central differences of the definition in 64 bits
    p = problem(31, torch.float16, 1, 100, 2, 1, 64, 64)
    q, k, v, decay, o, s, dout, dfinal = p
    got = tcr.linear_attention_backward(dout, q, k, v, decay, state=s, dfinal=dfinal)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)

    def loss(*ins):
        out, last, _, _ = definition(*ins[:3], decay, o, ins[3], 0.125)
        return ((out * dout.double()).sum() + (last * dfinal.double()).sum()).item()

    ins = [x.double() for x in (q, k, v, s)]
    for i in range(4):
        step = torch.randn(ins[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        up, down = list(ins), list(ins)
        up[i], down[i] = ins[i] + 1e-4 * step, ins[i] - 1e-4 * step
        want = (loss(*up) - loss(*down)) / 2e-4
        # the loss is linear in each input; the gradient's entries are rounded by 2^-11 at most, independently
        g = got[i].double()
        assert abs((g * step).sum().item() - want) <= 8 * 2.0 ** -12 * (g * step).norm().item() + 1e-6 * abs(want)


def test_repeatable_and_on_another_stream(tcr):
    p = problem(41, torch.bfloat16, 1, 3000, 4, 2, 128, 128)
    q, k, v, decay, o, s, dout, dfinal = p
    want = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
    grads = tcr.linear_attention_backward(dout, q, k, v, decay, state=s, dfinal=dfinal)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(tcr.linear_attention(q, k, v, decay, state=s, final_state=True), want))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
        more = tcr.linear_attention_backward(dout, q, k, v, decay, state=s, dfinal=dfinal)
    got2 = tcr.linear_attention(q, k, v, decay, state=s, final_state=True, stream=stream)
    stream.synchronize()
    for a, b, c in zip(got, got2, want):
        assert torch.equal(a, c) and torch.equal(b, c)
    assert all(torch.equal(a, b) for a, b in zip(more, grads))


def test_small_and_missing_workspaces(tcr):
    p = problem(43, torch.bfloat16, 1, 2500, 4, 2, 64, 64)
    q, k, v, decay, o, s, dout, dfinal = p
    u = HALF_SPACING[torch.bfloat16]
    want, last, size, last_size = definition(q, k, v, decay, o, s, 0.125)
    for n in (1 << 10, 1 << 18, 1 << 24):
        tcr.set_workspace(torch.empty(n, dtype=torch.uint8, device="cuda"))
        try:
            got, got_last = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
            near(got, want, size, u)
            near(got_last, last, last_size, 2.0 ** -19)
            if n < 1 << 20:
                with pytest.raises(tcr.TcrError) as e:
                    tcr.linear_attention_backward(dout, q, k, v, decay, state=s, dfinal=dfinal)
                assert e.value.status == tcr.ERR_WORKSPACE
        finally:
            tcr.set_workspace(None)
    check_gradients(tcr, p)


def test_recorded_into_a_graph(tcr):
    q, k, v, decay, o, s, dout, dfinal = problem(47, torch.float16, 1, 2000, 4, 4, 64, 64)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        tcr.linear_attention(q, k, v, decay, state=s, final_state=True)          # (the workspace)
        tcr.linear_attention_backward(dout, q, k, v, decay, state=s)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = tcr.linear_attention(q, k, v, decay, state=s, final_state=True)
        grads = tcr.linear_attention_backward(dout, q, k, v, decay, state=s)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    for _ in range(3):
        q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want, want_grads = tcr.linear_attention(q, k, v, decay, state=s, final_state=True), tcr.linear_attention_backward(dout, q, k, v, decay, state=s)
        u = HALF_SPACING[torch.float16]
        exact, last, size, last_size = definition(q, k, v, decay, o, s, 0.125)
        near(out[0], exact, size, u)
        near(out[1], last, last_size, 2.0 ** -19)
        assert all(torch.equal(a, b) for a, b in zip((*out, *grads), (*want, *want_grads)))


def test_long_offsets_beyond_32_bits(tcr):
    # the second sequence's rows start more than 2^32 bytes behind the first's
    heads, tokens, d = 2, 130, 64
    q, k, v, decay, o, s, dout, dfinal = problem(53, torch.bfloat16, 2, tokens, heads, heads, d, d)
    far = []
    for x in (q, k, v):
        room = torch.empty((1 << 31) + (1 << 20) + x[0].numel(), dtype=torch.bfloat16, device="cuda")
        w = room.as_strided(x.shape, ((1 << 31) + (1 << 20), heads * d, d, 1))
        w.copy_(x)
        far.append(w)
    want = tcr.linear_attention(q, k, v, decay, state=s)
    assert torch.equal(tcr.linear_attention(*far, decay, state=s), want)
    del far, room, w
    torch.cuda.empty_cache()                 # (12 GiB that later tests in this process may want to see free)


def test_refusals(tcr):
    q, k, v, decay, o, s, dout, dfinal = problem(61, torch.float16, 2, 10, 4, 2, 64, 64)
    call = tcr.linear_attention
    for bad in (lambda: call(q.cpu(), k, v, decay), lambda: call(q.float(), k.float(), v.float(), decay), lambda: call(q, k.bfloat16(), v, decay),
                lambda: call(q, k, v, decay.double()), lambda: call(q, k, v, decay[:3]), lambda: call(q, k, v, decay, state=s[:1]),
                lambda: call(q, k, v, decay, state=s.half()), lambda: call(q[..., ::2], k[..., ::2], v, decay),
                lambda: call(q[0], k[0], v[0], decay), lambda: call(q, k, v, decay, offsets=torch.zeros(3, dtype=torch.int64, device="cuda")),
                lambda: call(q[0], k[0], v[0], decay, offsets=torch.zeros(3, dtype=torch.int32, device="cuda")),
                lambda: tcr.linear_attention_step(q, k, v, decay, s), lambda: tcr.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, s[..., ::2])):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: call(q, k[:, :, :1].expand(-1, -1, 3, -1), v[:, :, :1].expand(-1, -1, 3, -1), decay), lambda: call(q, k[:, :5], v[:, :5], decay),
                lambda: call(q, k[..., :32], v, decay), lambda: call(q, k, v[:, :, :1], decay)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: call(q[..., :60], k[..., :60], v, decay), tcr.ERR_UNSUPPORTED), (lambda: call(q, k, v, decay, scale=0.0), tcr.ERR_INVALID_ARG),
                        (lambda: call(q, k, v, decay, scale=float("nan")), tcr.ERR_INVALID_ARG)):
        with pytest.raises(tcr.TcrError) as e:
            bad()
        assert e.value.status == status

"""Linear attention where sequences meet: values without a number stay in their sequence, whatever blocks and kernels the tokens are cut into;
tokens outside every sequence, offsets that are none, and results that do not depend on what else is asked for."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tcr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1811_09736_amd import binding
    return binding


def inputs(seed, lead, heads, kv, d, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    make = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    return make(*lead, heads, d), make(*lead, kv, d), make(*lead, kv, d), -0.01 * torch.rand(heads, generator=gen, device="cuda"), make(*lead, heads, d)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("batch,tokens,heads,kv", [(3, 2, 4, 4), (4, 100, 2, 2), (3, 700, 2, 1), (2, 3000, 2, 2), (5, 1100, 8, 8)])
def test_other_sequences_do_not_notice(tcr, bad, dtype, batch, tokens, heads, kv):
    q, k, v, decay, do = inputs(1, (batch, tokens), heads, kv, 64, dtype)
    want = tcr.linear_attention(q, k, v, decay, final_state=True)
    grads = tcr.linear_attention_backward(do, q, k, v, decay)[:3]
    for at in (k, v):
        spoilt = at.clone()
        spoilt[1, tokens // 2, 0, 3] = bad
        a, b = (spoilt, v) if at is k else (k, spoilt)
        out, last = tcr.linear_attention(q, a, b, decay, final_state=True)
        others = [i for i in range(batch) if i != 1]
        assert torch.equal(out[others], want[0][others]) and torch.equal(last[others], want[1][others])
        assert not torch.isfinite(out[1, tokens // 2:]).all()
        # the spoilt sequence's earlier tokens too, but for the 63 in front
        early = max(0, tokens // 2 - 63)
        assert torch.equal(out[1, :early], want[0][1, :early])
        for g, w in zip(tcr.linear_attention_backward(do, q, a, b, decay)[:3], grads):
            assert torch.equal(g[others], w[others])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_other_packed_sequences_do_not_notice(tcr, dtype):
    cuts = [0, 400, 401, 401, 1500, 4000]
    q, k, v, decay, do = inputs(2, (4000,), 4, 2, 64, dtype)
    o = torch.tensor(cuts, device="cuda")
    want = tcr.linear_attention(q, k, v, decay, offsets=o, final_state=True)
    grads = tcr.linear_attention_backward(do, q, k, v, decay, offsets=o)[:3]
    spoilt = v.clone()
    spoilt[700, 1, 5] = float("nan")
    out, last = tcr.linear_attention(q, k, spoilt, decay, offsets=o, final_state=True)
    keep = torch.ones(4000, dtype=torch.bool, device="cuda")
    keep[401:1500] = False
    assert torch.equal(out[keep], want[0][keep]) and torch.equal(last[[0, 1, 2, 4]], want[1][[0, 1, 2, 4]]) and torch.isnan(out[700:1500]).any()
    for g, w in zip(tcr.linear_attention_backward(do, q, k, spoilt, decay, offsets=o)[:3], grads):
        assert torch.equal(g[keep], w[keep])


@pytest.mark.parametrize("first,last", [(0, 300), (5000, 5300), (9700, 10000), (4000, 4001), (10000, 10000), (0, 0)])
def test_few_sequences_in_a_large_buffer(tcr, first, last):
    total = 10000
    q, k, v, decay, do = inputs(3, (total,), 2, 2, 64, torch.bfloat16)
    middle = (first + last) // 2
    o = torch.tensor([first, middle, last], device="cuda")
    out, state = tcr.linear_attention(q, k, v, decay, offsets=o, final_state=True)
    grads = tcr.linear_attention_backward(do, q, k, v, decay, offsets=o)[:3]
    inside = torch.arange(first, last, device="cuda")
    if last > first:
        ref, ref_state = tcr.linear_attention(q[first:last], k[first:last], v[first:last], decay, offsets=o - first, final_state=True)
        # (cut into other blocks: other roundings of sums in 32 bits, then one to bfloat16)
        assert (out[inside].float() - ref.float()).norm() <= 2.0 ** -8 * ref.float().norm()
        assert (state - ref_state).norm() <= 1e-5 * ref_state.norm()
    for x in (out, *grads):
        rest = torch.ones(total, dtype=torch.bool, device="cuda")
        rest[inside] = False
        assert (x[rest] == 0).all() and torch.isfinite(x).all()
    assert torch.isfinite(state).all()


@pytest.mark.parametrize("offsets", [[0, 500, 100, 900], [900, 400, 100, 0], [0, 1 << 40, 1 << 41, 5], [3, 3, 3, 3], [-5, 10, -1, 900]])
def test_offsets_that_are_none_end_quietly(tcr, offsets):
    # wrong numbers, but every call comes back and later ones are right
    q, k, v, decay, do = inputs(4, (900,), 2, 2, 64, torch.float16)
    guard = torch.full((900 * 2 * 64 + 256,), 7.0, dtype=torch.float16, device="cuda")
    out = guard[128:-128].view(900, 2, 64)
    tcr.linear_attention(q, k, v, decay, offsets=torch.tensor(offsets, device="cuda"), final_state=True, out=out)
    tcr.linear_attention_backward(do, q, k, v, decay, offsets=torch.tensor(offsets, device="cuda"))
    torch.cuda.synchronize()
    assert (guard[:128] == 7).all() and (guard[-128:] == 7).all()
    o = torch.tensor([0, 900], device="cuda")
    a, b = tcr.linear_attention(q, k, v, decay, offsets=o), tcr.linear_attention(q[None], k[None], v[None], decay)[0]
    assert (a.float() - b.float()).norm() <= 2.0 ** -10 * b.float().norm()


def test_given_outputs_and_views(tcr):
    q, k, v, decay, do = inputs(5, (2, 300), 4, 4, 128, torch.bfloat16)
    want = tcr.linear_attention(q, k, v, decay)
    # q, k, v as parts of one projection's rows
    rows = torch.cat([q.flatten(2), k.flatten(2), v.flatten(2)], -1)
    a, b, c = rows.unflatten(-1, (3, 4, 128)).unbind(2)
    assert torch.equal(tcr.linear_attention(a, b, c, decay), want)
    assert all(torch.equal(x, y) for x, y in zip(tcr.linear_attention_backward(do, a, b, c, decay)[:3], tcr.linear_attention_backward(do, q, k, v, decay)[:3]))

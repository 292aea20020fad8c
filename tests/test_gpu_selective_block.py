"""The example of examples/selective_block.py: gradients against plain torch in 64 bits, a training step with clipping, serving that gives what the model gives; graphs and
streams over a run of its operators."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def block():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("selective_block", os.path.join(ROOT, "examples", "selective_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(model, tokens, p):
    """The model's logits in 64 bits by elementary operations."""
    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w

    total, y = p["embedding"][tokens], None
    for i, block in enumerate(model.blocks):
        get = lambda n: p[f"blocks.{i}.{n}"]  # noqa: B023, E731
        total = total if y is None else total + y
        x, z = (norm(total, get("norm")) @ get("into").T).chunk(2, -1)
        taps = get("taps")
        width = taps.shape[1]
        front = torch.cat([x.new_zeros(x.shape[0], width - 1, x.shape[2]), x], 1)
        h = sum(front[:, j:j + x.shape[1]] * taps[:, j] for j in range(width)) + get("taps_bias")
        h = h / (1 + torch.exp(-h))
        dt, b, c = (h @ get("select").T).split((block.rank, block.states, block.states), -1)
        d = torch.log1p(torch.exp(dt @ get("step").T + get("step_bias")))
        a = -get("log_rate").exp()
        s, ys = h.new_zeros(h.shape[0], h.shape[2], block.states), []
        for t in range(h.shape[1]):
            s = torch.exp(d[:, t, :, None] * a) * s + (d[:, t] * h[:, t])[..., None] * b[:, t, None]
            ys.append((s * c[:, t, None]).sum(2))
        out = (torch.stack(ys, 1) + get("skip") * h) * z / (1 + torch.exp(-z))
        y = out @ get("back").T
    return norm(total + y, p["norm"]) @ p["head"].T


def test_gradients_of_the_whole_model(block):
    torch.manual_seed(1)
    model = block.Model(vocabulary=32, width=32, inner=64, states=8, blocks=2)
    tokens = torch.randint(0, 32, (3, 50), device="cuda")
    target = torch.randn(3, 50, 32, device="cuda")
    logits = model(tokens)
    (logits.float() * target).sum().backward()
    parameters = {n: p.detach().double().requires_grad_() for n, p in model.named_parameters()}
    want = plain(model, tokens, parameters)
    (want * target.double()).sum().backward()
    # every activation on the way is rounded to bfloat16, 2^-9 relative on average: two blocks of about ten roundings each
    assert (logits.double() - want).norm() <= 0.04 * want.norm()
    for n, p in model.named_parameters():
        assert p.grad is not None and (p.grad.double() - parameters[n].grad).norm() <= 0.08 * parameters[n].grad.norm(), n


def test_a_training_step_clips_all_gradients_together(block):
    torch.manual_seed(0)
    model = block.Model(blocks=1)
    losses, norms = block.train(model, 3, limit=0.5)
    assert len(losses) == 3 and all(n > 0 and n == n for n in norms)
    # what the last step left clipped: half the limit's own rounding, bfloat16's half step for most elements
    from paper_1811_09736_amd import binding
    left = float(binding.gradient_norm([p.grad for p in model.parameters()]))
    assert left <= (1 + 2.0 ** -8) * min(0.5, norms[-1])


def test_serving_goes_on_like_the_prompt(block):
    torch.manual_seed(2)
    model = block.Model()
    sequences = [torch.randint(0, 64, (n,), device="cuda") for n in (37, 1, 80)]
    whole = torch.tensor([0, 37, 38, 118], device="cuda")
    want = model.serve(torch.cat(sequences), model.states(3), whole)
    # all but the last token as prompts (one of them empty), the last as a step
    heads = torch.tensor([0, 36, 36, 115], device="cuda")
    states = model.states(3)
    first = model.serve(torch.cat([s[:-1] for s in sequences]), states, heads)
    last = model.serve(torch.stack([s[-1] for s in sequences]), states)
    kept = torch.cat([torch.arange(0, 36), torch.arange(38, 117)]).cuda()
    # the same operations on the same values but for the order of sums, whose rounding may move a bfloat16 value by a step here and there
    assert (first.float() - want[kept].float()).norm() <= 0.02 * want.float().norm()
    assert (last.float() - want[whole[1:] - 1].float()).norm() <= 0.02 * want[whole[1:] - 1].float().norm()


def test_partial_gradients(block):
    from paper_1811_09736_amd import autograd
    x = torch.randn(2, 20, 24, device="cuda", requires_grad=True)
    w = torch.randn(24, 4, device="cuda", requires_grad=True)
    out, last = autograd.causal_conv(x, w)
    last.sum().backward()                                       # only the last inputs are used
    assert (x.grad[:, :17] == 0).all() and (x.grad[:, 17:] == 1).all() and (w.grad == 0).all()
    dt, a = torch.randn(2, 20, 24, device="cuda", requires_grad=True), -torch.rand(24, 4, device="cuda")
    b, c = torch.randn(2, 20, 1, 4, device="cuda"), torch.randn(2, 20, 1, 4, device="cuda", requires_grad=True)
    state = torch.randn(2, 24, 4, device="cuda", requires_grad=True)
    out, last = autograd.selective_scan(x.detach(), dt, a, b, c, state=state)
    last.sum().backward()
    d = torch.nn.functional.softplus(dt.detach()).sum(1)
    # (the exponent's own error counts: up to 60 here, 2^-24 of it for each of 20 sums)
    assert (c.grad == 0).all() and torch.allclose(state.grad, torch.exp(d[..., None] * a), rtol=1e-4, atol=1e-7) and dt.grad.abs().sum() > 0
    with pytest.raises(RuntimeError):
        grad, = torch.autograd.grad(autograd.causal_conv(x, w)[0].sum(), x, create_graph=True)
        grad.sum().backward()


def run(tcr, v):
    """A block's operators one behind the other, forwards and backwards, and the clipping."""
    h, last = tcr.causal_conv(v["x"], v["w"], v["bias"], state=v["front"], final_state=True)
    out, end = tcr.selective_scan(h, v["dt"], v["a"], v["b"], v["c"], skip=v["skip"], gate=v["gate"], dt_bias=v["dt_bias"], state=v["state"], final_state=True)
    grads = tcr.selective_scan_backward(v["dout"], h, v["dt"], v["a"], v["b"], v["c"], skip=v["skip"], gate=v["gate"], dt_bias=v["dt_bias"], state=v["state"])
    more = tcr.causal_conv_backward(grads[0], v["x"], v["w"], v["bias"], state=v["front"])
    wanted = [*grads, *more]
    norm = tcr.clip_gradients(wanted, 1.0)
    step = tcr.causal_conv_step(v["x"][:, 0], v["w"], last, v["bias"])
    token = tcr.selective_scan_step(step, v["dt"][:, 0], v["a"], v["b"][:, 0], v["c"][:, 0], end, skip=v["skip"], gate=v["gate"][:, 0], dt_bias=v["dt_bias"])
    return [h, last, out, end, norm, step, token, *wanted]


def make(seed, tokens=300, channels=96):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    half = lambda *s: r(*s).to(torch.bfloat16)  # noqa: E731
    return {"x": half(2, tokens, channels), "w": half(channels, 4), "bias": half(channels), "front": half(2, 3, channels), "dt": half(2, tokens, channels),
            "a": -torch.rand(channels, 16, generator=gen, device="cuda") * 4, "b": half(2, tokens, 1, 16), "c": half(2, tokens, 1, 16), "skip": r(channels),
            "gate": half(2, tokens, channels), "dt_bias": r(channels) - 2, "state": r(2, channels, 16), "dout": half(2, tokens, channels)}


def test_a_captured_run_replays(block):
    from paper_1811_09736_amd import binding as tcr
    held, other = make(0), make(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(tcr, held)                                          # the workspace of the stream is there before it is recorded
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run(tcr, held)
    for seed in (1, 2, 3):
        fresh = make(seed)
        for k in held:
            held[k].copy_(fresh[k])
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        want = run(tcr, fresh)                                  # (eager work between the replays)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(kept, want))
    del other


def test_a_recorded_call_without_workspace_is_refused(block):
    from paper_1811_09736_amd import binding as tcr
    v = make(4)
    fresh = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    fresh.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=fresh):
        out = tcr.selective_scan(v["x"], v["dt"], v["a"], v["b"], v["c"])           # fewer chunks, without workspace
        with pytest.raises(tcr.TcrError):
            tcr.selective_scan_backward(v["dout"], v["x"], v["dt"], v["a"], v["b"], v["c"])
        with pytest.raises(tcr.TcrError):
            tcr.causal_conv_backward(v["dout"], v["x"], v["w"])
        with pytest.raises(tcr.TcrError):
            tcr.clip_gradients([v["skip"]], 1.0)
    graph.replay()
    torch.cuda.synchronize()
    want = tcr.selective_scan(v["x"], v["dt"], v["a"], v["b"], v["c"])
    # (other chunks, other roundings in binary32: at most a step of bfloat16)
    assert ((out.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-4).all()


def test_two_streams_at_once(block):
    from paper_1811_09736_amd import binding as tcr
    inputs = [make(seed, tokens=700) for seed in (5, 6)]
    want = [run(tcr, v) for v in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    got = []
    for _ in range(3):
        got = []
        for v, s in zip(inputs, streams):
            with torch.cuda.stream(s):
                got.append(run(tcr, v))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))


def test_a_callers_workspace(block):
    from paper_1811_09736_amd import binding as tcr
    v = make(7)
    want = run(tcr, v)
    torch.cuda.synchronize()
    small, large = torch.empty(4096, dtype=torch.uint8, device="cuda"), torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    try:
        tcr.set_workspace(large)
        assert all(torch.equal(p, q) for p, q in zip(run(tcr, v), want))
        tcr.set_workspace(small)
        out = tcr.selective_scan(v["x"], v["dt"], v["a"], v["b"], v["c"])
        before = v["dout"].clone()
        with pytest.raises(tcr.TcrError) as e:
            tcr.selective_scan_backward(v["dout"], v["x"], v["dt"], v["a"], v["b"], v["c"])
        assert e.value.status == tcr.ERR_WORKSPACE and torch.equal(before, v["dout"])
    finally:
        tcr.set_workspace(None)
    usual = tcr.selective_scan(v["x"], v["dt"], v["a"], v["b"], v["c"])
    assert ((out.float() - usual.float()).abs() <= 2.0 ** -7 * usual.float().abs() + 1e-4).all()

"""The selective state space scan with its short causal convolution (prompts, their gradients, single tokens) and the gradient norm
over many tensors with the clipping, as cases that can be timed and compared: each in its plain form, elementary torch operations in
32 bits, and through the library's calls.

A case is a dict of plain values:

  op        "conv", "conv_backward", "conv_step", "scan", "scan_backward", "scan_step", "clip"
  dtype     "bf16", "f16" or "f32": the type of inputs and outputs; states of the scan, its rates and biases are binary32
  conv, scan: batch x tokens (or `seqs` packed sequences of `tokens` tokens in all; a step: one token for each of `batch`), channels;
            state: whether the sequences go on from given states
  conv:     width (taps), act: whether silu follows
  scan:     states (a channel's), groups (of channels that share b and c), gate: whether the output is gated
  clip:     blocks x the tensors of a block of width `channels`; clips: whether the norm lies above the limit
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # a long prompt on its way into the scan
        {"name": "conv_prompt", "op": "conv", "dtype": "bf16", "seqs": 0, "batch": 1, "tokens": 16384, "channels": 4096, "width": 4, "act": True,
         "state": False},
        # a training step's packed sequences, an empty one and one of a single token among them
        {"name": "conv_grad_packed", "op": "conv_backward", "dtype": "f16", "seqs": 9, "batch": 1, "tokens": 8191, "channels": 4096, "width": 4,
         "act": True, "state": False},
        # the next token of a full batch
        {"name": "conv_step_256", "op": "conv_step", "dtype": "bf16", "batch": 256, "channels": 4096, "width": 4, "act": True},
        # one long prompt
        {"name": "scan_prompt", "op": "scan", "dtype": "bf16", "seqs": 0, "batch": 1, "tokens": 8192, "channels": 4096, "states": 16, "groups": 1,
         "gate": True, "state": False},
        # prompts of different lengths packed behind one another that go on from earlier parts, b and c by groups of channels
        {"name": "scan_packed", "op": "scan", "dtype": "f16", "seqs": 13, "batch": 1, "tokens": 8191, "channels": 2048, "states": 16, "groups": 2,
         "gate": True, "state": True},
        # a short question
        {"name": "scan_short", "op": "scan", "dtype": "bf16", "seqs": 0, "batch": 1, "tokens": 173, "channels": 2048, "states": 16, "groups": 1,
         "gate": True, "state": False},
        # the gradients of one training step's sequences
        {"name": "scan_grad_4x2048", "op": "scan_backward", "dtype": "bf16", "seqs": 0, "batch": 4, "tokens": 2048, "channels": 2048, "states": 16,
         "groups": 1, "gate": True, "state": False},
        # the same for packed sequences, a number of channels that no vector divides, few states
        {"name": "scan_grad_odd", "op": "scan_backward", "dtype": "f16", "seqs": 9, "batch": 1, "tokens": 1531, "channels": 1001, "states": 7,
         "groups": 1, "gate": False, "state": True},
        # one conversation's next token: latency
        {"name": "scan_step_1", "op": "scan_step", "dtype": "bf16", "batch": 1, "channels": 4096, "states": 16, "groups": 1, "gate": True},
        # the next token of a full batch: the states' bytes
        {"name": "scan_step_256", "op": "scan_step", "dtype": "f16", "batch": 256, "channels": 4096, "states": 16, "groups": 1, "gate": True},
        # a small model's gradients: latency
        {"name": "clip_small", "op": "clip", "dtype": "bf16", "blocks": 4, "channels": 256, "clips": True},
        # a large one's, in binary32
        {"name": "clip_large", "op": "clip", "dtype": "f32", "blocks": 32, "channels": 1024, "clips": True},
    ]


def _size(rng, low, high):
    """A size between the two, evenly over its logarithm: a power of two a third of the time, odd otherwise."""
    v = 2.0 ** rng.uniform(math.log2(low), math.log2(high))
    return max(low, min(1 << round(math.log2(v)) if rng.random() < 0.33 else int(v) | 1, high))


def draw(rng):
    op = rng.choice(("conv", "conv_backward", "conv_step", "scan", "scan", "scan", "scan_backward", "scan_backward", "scan_step", "clip"))
    case = {"op": op, "dtype": rng.choice(("bf16", "bf16", "f16", "f32"))}
    if op == "clip":
        case["channels"] = _size(rng, 32, 1024)
        case["blocks"] = _size(rng, 1, min(64, (96 << 20) // (3 * case["channels"] ** 2)))
        case["clips"] = rng.random() < 0.7
        return case
    case["channels"] = rng.choice((1024, 1536, 2048, 2560, 4096)) if rng.random() < 0.6 else _size(rng, 24, 4096)
    if op.startswith("conv"):
        case["width"], case["act"] = rng.choice((2, 3, 4, 4)), rng.random() < 0.8
        limit = 1 << 25
    else:
        case["states"] = rng.choice((16, 16, 16, 8, 32, 64, 4, 7, 12, 1))
        case["groups"] = 2 if case["channels"] % 2 == 0 and rng.random() < 0.3 else 1
        case["gate"] = rng.random() < 0.7
        limit = (1 << 28 if op == "scan" else 1 << 27) // case["states"]
    if op.endswith("step"):
        case["batch"] = _size(rng, 1, min(512, limit // case["channels"]))
        return case
    case["seqs"] = rng.choice((0, 0, 5, 13))
    case["batch"] = 1 if case["seqs"] else rng.choice((1, 2, 4))
    limit = min(limit // case["channels"] // case["batch"], 8192)
    case["tokens"] = _size(rng, 1 if not case["seqs"] else min(512, limit), limit)
    case["state"] = rng.random() < 0.4
    return case


def _lengths(case, gen):
    """Offsets of the packed sequences: one empty, one of a single token, the others of different lengths."""
    n, total = case["seqs"], case["tokens"]
    share = torch.rand(n - 2, generator=gen, device=gen.device, dtype=torch.float64) + 0.1
    ends = torch.floor(torch.cumsum(share, 0) / share.sum() * (total - 1)).to(torch.int64)
    ends[-1] = total - 1
    first = ends[:1]
    # (the empty sequence stands second, the single token third)
    return torch.cat([first.new_zeros(1), first, first, first + 1, ends[1:] + 1])


def _shapes(case):
    """A model's parameters: of every block the projections, the short convolution, what the scan has, the norm; matrices, and
    vectors that are kept in binary32 whatever the matrices are."""
    c = case["channels"]
    block = [(c, 2 * c), (c, 4), (c,), (c, 16), (c, c + 33), (c,), (c,), (c // 2,)]
    return block * case["blocks"] + [(1000, c), (c,)]


def _buckets(tensors):
    """Flat tensors of zeros, one for each type among `tensors`, and the place of each tensor in them, on a boundary of 8 elements."""
    at, sizes = [], {}
    for t in tensors:
        at.append(sizes.get(t.dtype, 0))
        sizes[t.dtype] = at[-1] + -(-t.numel() // 8) * 8
    flat = {dtype: torch.zeros(size, dtype=dtype, device="cuda") for dtype, size in sizes.items()}
    return tuple(flat.values()), [flat[t.dtype][first:first + t.numel()].view(t.shape) for t, first in zip(tensors, at)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = _TYPES[case["dtype"]]

    def normal(*shape, spread=1.0, dtype=dtype):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * spread).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda", dtype=torch.float32)

    state = dict(case)
    if case["op"] == "clip":
        shapes = _shapes(case)
        state["grads"] = [normal(*s, spread=0.01, dtype=dtype if len(s) == 2 else torch.float32) for s in shapes]
        # what is clipped goes to the buckets that the optimizer reads, one for each type (a pass can be repeated: the gradients stay)
        state["buckets"], state["clipped"] = _buckets(state["grads"])
        state["limit"] = 0.01 * math.sqrt(sum(math.prod(s) for s in shapes)) * (0.4 if case["clips"] else 2.5)
        return state
    channels = case["channels"]
    step = case["op"].endswith("step")
    packed = not step and case["seqs"] > 0
    lead = (case["batch"],) if step else (case["tokens"],) if packed else (case["batch"], case["tokens"])
    count = case["seqs"] if packed else case["batch"]
    if not step:
        state["offsets"] = _lengths(case, gen) if packed else None
        state["longest"] = int((state["offsets"][1:] - state["offsets"][:-1]).max()) if packed else case["tokens"]
    # x is one part of a projection's rows, the gate the other
    both = normal(*lead, 2 * channels)
    state["x"] = both[..., :channels]
    if case["op"].startswith("conv"):
        width = case["width"]
        state["weight"], state["bias"] = normal(channels, width, spread=width ** -0.5), normal(channels, spread=0.2)
        state["s"] = normal(count, width - 1, channels) if step or case["state"] else None
        state["dfinal"] = normal(count, width - 1, channels) if case["op"] == "conv_backward" and case["state"] else None
    else:
        n, groups = case["states"], case["groups"]
        state["gate_in"] = both[..., channels:] if case["gate"] else None
        # steps between a thousandth and a tenth, rates from 1 to the number of states
        state["dt"] = normal(*lead, channels, spread=0.5)
        target = torch.exp(uniform(channels) * math.log(100.0) + math.log(1e-3))
        state["dt_bias"] = target + torch.log(-torch.expm1(-target))
        state["a"] = -torch.arange(1, n + 1, device="cuda", dtype=torch.float32) * (0.8 + 0.4 * uniform(channels, n))
        state["b"], state["c"] = normal(*lead, groups, n), normal(*lead, groups, n)
        state["skip"] = 1.0 + normal(channels, spread=0.1, dtype=torch.float32)
        state["s"] = normal(count, channels, n, dtype=torch.float32) if step or case["state"] else None
        state["dfinal"] = normal(count, channels, n, dtype=torch.float32) if case["op"] == "scan_backward" and case["state"] else None
    if step:
        state["next"] = torch.empty_like(state["s"])       # (a pass can be repeated: the new state stands beside the old one)
    if case["op"].endswith("backward"):
        state["dout"] = normal(*lead, channels)
    return state


# ------------------------------------------------------------------------------------------------ plain forms
def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _softplus(x):
    """log(1 + exp(x)), without loss where exp(x) is small."""
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def _rows(x, state):
    """[sequences, longest, ...] in 32 bits, every sequence at the start of its row, zeros behind."""
    x = x.float()
    if state["offsets"] is None:
        return x
    o = state["offsets"]
    at = o[:-1, None] + torch.arange(state["longest"], device=x.device)
    inside = (at < o[1:, None]).view(*at.shape, *(1,) * (x.dim() - 1))
    return torch.where(inside, x[at.clamp(max=x.shape[0] - 1)], 0.0)


def _lens(state):
    if state["offsets"] is None:
        return torch.full((state["batch"],), state["tokens"], device=state["x"].device)
    return state["offsets"][1:] - state["offsets"][:-1]


def _back(x, state):
    """The inverse of _rows."""
    if state["offsets"] is None:
        return x
    o = state["offsets"]
    at = torch.arange(state["tokens"], device=x.device)
    seq = torch.searchsorted(o[1:], at, right=True)
    return x[seq, at - o[seq]]


def _conv_sums(state):
    """The inputs with the width - 1 in front of each sequence, and the sums in front of the activation."""
    x, w = _rows(state["x"], state), state["weight"].float()
    width = state["width"]
    front = state["s"].float() if state["s"] is not None else x.new_zeros(x.shape[0], width - 1, x.shape[2])
    x = torch.cat([front, x], 1)
    length = x.shape[1] - width + 1
    return x, sum(x[:, j:j + length] * w[:, j] for j in range(width)) + state["bias"].float()


def _plain_conv(state):
    x, s = _conv_sums(state)
    y = s * _sigmoid(s) if state["act"] else s
    at = _lens(state)[:, None] + torch.arange(state["width"] - 1, device=x.device)
    last = torch.gather(x, 1, at[..., None].expand(-1, -1, x.shape[2]))
    dtype = state["x"].dtype
    return _back(y, state).to(dtype), last.to(dtype)


def _plain_conv_backward(state):
    x, s = _conv_sums(state)
    w, width, dtype = state["weight"].float(), state["width"], state["x"].dtype
    ds = _rows(state["dout"], state)
    length = ds.shape[1]
    if state["act"]:
        g = _sigmoid(s)
        ds = ds * (g + s * g * (1.0 - g))
    dx = torch.zeros_like(x)
    for j in range(width):
        dx[:, j:j + length] += ds * w[:, j]
    if state["dfinal"] is not None:
        at = _lens(state)[:, None] + torch.arange(width - 1, device=x.device)
        dx.scatter_add_(1, at[..., None].expand(-1, -1, x.shape[2]), state["dfinal"].float())
    dw = torch.stack([(ds * x[:, j:j + length]).sum((0, 1)) for j in range(width)], 1)
    got = (_back(dx[:, width - 1:], state).to(dtype), dw.to(dtype), ds.sum((0, 1)).to(dtype))
    return got if state["s"] is None else (*got, dx[:, :width - 1].to(dtype))


def _plain_conv_step(state):
    x = torch.cat([state["s"].float(), state["x"].float()[:, None]], 1)
    s = (x * state["weight"].float().T).sum(1) + state["bias"].float()
    y = s * _sigmoid(s) if state["act"] else s
    return y.to(state["x"].dtype), x[:, 1:].to(state["x"].dtype)


def _running(keep, add, h):
    """h_t = keep_t h_{t-1} + add_t along the second axis, all of them in the place of add."""
    for t in range(add.shape[1]):
        h = torch.addcmul(add[:, t], keep[:, t], h, out=add[:, t])
    return add


def _scan_inputs(state):
    """x, dt in front of and behind the softplus (0 behind a sequence's end), b and c for every channel."""
    x = _rows(state["x"], state)
    raw = _rows(state["dt"], state) + state["dt_bias"]
    inside = torch.arange(state["longest"], device=x.device) < _lens(state)[:, None]
    dt = torch.where(inside[..., None], _softplus(raw), 0.0)
    return x, raw, dt, _rows(state["b"], state), _rows(state["c"], state)


def _spread(x, channels):
    """[..., groups, n] for every channel: [..., channels, n]."""
    if x.shape[-2] == 1:
        return x
    return x.repeat_interleave(channels // x.shape[-2], -2)


def _plain_scan(state):
    x, _, dt, b, c = _scan_inputs(state)
    a, channels = state["a"], state["channels"]
    h = state["s"] if state["s"] is not None else x.new_zeros(x.shape[0], channels, state["states"])
    y = torch.empty_like(x)
    size = max(1, (1 << 26) // h.numel())
    for top in range(0, x.shape[1], size):
        part = slice(top, top + size)
        add = (dt * x)[:, part, :, None] * _spread(b[:, part], channels)
        hs = _running(torch.exp(dt[:, part, :, None] * a), add, h)
        h = hs[:, -1].clone()
        y[:, part] = (hs * _spread(c[:, part], channels)).sum(3)
    y = y + state["skip"] * x
    if state["gate"]:
        z = _rows(state["gate_in"], state)
        y = y * z * _sigmoid(z)
    return _back(y, state).to(state["x"].dtype), h


def _plain_scan_backward(state):
    x, raw, dt, b, c = _scan_inputs(state)
    a, channels, groups, dtype = state["a"], state["channels"], state["groups"], state["x"].dtype
    length = x.shape[1]
    h0 = state["s"] if state["s"] is not None else x.new_zeros(x.shape[0], channels, state["states"])
    keep = torch.exp(dt[..., None] * a)
    hs = torch.empty_like(keep)
    torch.mul((dt * x)[..., None], _spread(b, channels), out=hs)
    _running(keep, hs, h0)
    y = torch.stack([(hs[:, t] * _spread(c[:, t], channels)).sum(2) for t in range(length)], 1) + state["skip"] * x
    dy = _rows(state["dout"], state)
    dz = None
    if state["gate"]:
        z = _rows(state["gate_in"], state)
        s = _sigmoid(z)
        dz = dy * y * (s + z * s * (1.0 - s))
        dy = dy * z * s
    grad = state["dfinal"].clone() if state["dfinal"] is not None else torch.zeros_like(h0)
    db, dc, ddt, dx = torch.empty_like(b), torch.empty_like(c), torch.empty_like(dt), dy * state["skip"]
    da = torch.zeros_like(a)
    for t in range(length - 1, -1, -1):
        bt, step = _spread(b[:, t], channels), dt[:, t, :, None]
        grad = grad + dy[:, t, :, None] * _spread(c[:, t], channels)
        dc[:, t] = (dy[:, t, :, None] * hs[:, t]).unflatten(1, (groups, -1)).sum(2)
        db[:, t] = (grad * (step * x[:, t, :, None])).unflatten(1, (groups, -1)).sum(2)
        gb = (grad * bt).sum(2)
        grad = grad * keep[:, t]
        back = grad * (hs[:, t - 1] if t > 0 else h0)
        dx[:, t] += gb * dt[:, t]
        ddt[:, t] = gb * x[:, t] + (back * a).sum(2)
        da += (back * step).sum(0)
    inside = (torch.arange(length, device=x.device) < _lens(state)[:, None])[..., None]
    ddt = torch.where(inside, ddt * _sigmoid(raw), 0.0)
    got = (_back(dx, state).to(dtype), _back(ddt, state).to(dtype), da, _back(db, state).to(dtype), _back(dc, state).to(dtype),
           (dy * x).sum((0, 1)))
    if state["gate"]:
        got += (_back(dz, state).to(dtype),)
    got += (ddt.sum((0, 1)),)
    return got if state["s"] is None else (*got, grad)


def _plain_scan_step(state):
    x, dt = state["x"].float(), _softplus(state["dt"].float() + state["dt_bias"])
    b, c = _spread(state["b"].float(), state["channels"]), _spread(state["c"].float(), state["channels"])
    h = torch.exp(dt[..., None] * state["a"]) * state["s"] + (dt * x)[..., None] * b
    y = (h * c).sum(2) + state["skip"] * x
    if state["gate"]:
        z = state["gate_in"].float()
        y = y * z * _sigmoid(z)
    return y.to(state["x"].dtype), h


def _plain_clip(state):
    # (squares of sums over many tensors: in 64 bits)
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in state["grads"]]).sum().sqrt().float()
    factor = (state["limit"] / (norm + 1e-6)).clamp(max=1.0)
    for g, to in zip(state["grads"], state["clipped"]):
        to.copy_(g.float() * factor)
    return (norm, *state["buckets"])


# ------------------------------------------------------------------------------------------------ the library's calls
def _own(state):
    from paper_1811_09736_amd import binding
    op = state["op"]
    if op == "clip":
        return (binding.clip_gradients(state["grads"], state["limit"], out=state["clipped"]), *state["buckets"])
    if op.startswith("conv"):
        given = {"bias": state["bias"], "activation": "silu" if state["act"] else None}
        if op == "conv":
            return binding.causal_conv(state["x"], state["weight"], offsets=state["offsets"], state=state["s"], final_state=True, **given)
        if op == "conv_step":
            return binding.causal_conv_step(state["x"], state["weight"], state["s"], new_state=state["next"], **given), state["next"]
        got = binding.causal_conv_backward(state["dout"], state["x"], state["weight"], offsets=state["offsets"], state=state["s"],
                                           dfinal=state["dfinal"], **given)
        return tuple(g for g in got if g is not None)
    args = (state["x"], state["dt"], state["a"], state["b"], state["c"])
    given = {"skip": state["skip"], "gate": state["gate_in"], "dt_bias": state["dt_bias"]}
    if op == "scan":
        return binding.selective_scan(*args, offsets=state["offsets"], state=state["s"], final_state=True, **given)
    if op == "scan_step":
        return binding.selective_scan_step(*args, state["s"], new_state=state["next"], **given), state["next"]
    got = binding.selective_scan_backward(state["dout"], *args, offsets=state["offsets"], state=state["s"], dfinal=state["dfinal"], **given)
    return tuple(g for g in got if g is not None)


_PLAIN = {"conv": _plain_conv, "conv_backward": _plain_conv_backward, "conv_step": _plain_conv_step, "scan": _plain_scan,
          "scan_backward": _plain_scan_backward, "scan_step": _plain_scan_step, "clip": _plain_clip}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


def work(case):
    """Inputs read once, outputs written once (clipping: the gradients twice, as the norm of all of them comes first).  The scan by its
    recurrence: for each state and token a product with the rate, an exponential, two multiply-adds and the product with b."""
    op, e = case["op"], 4 if case["dtype"] == "f32" else 2
    if op == "clip":
        sizes = [(math.prod(s), e if len(s) == 2 else 4) for s in _shapes(case)]
        return {"bytes": 3 * sum(n * size for n, size in sizes) + 4, "flops": 3 * sum(n for n, _ in sizes)}
    channels = case["channels"]
    tokens = case["batch"] if op.endswith("step") else case["tokens"] * case["batch"]
    count = case["batch"] if op.endswith("step") else case["seqs"] or case["batch"]
    n = tokens * channels
    if op.startswith("conv"):
        weights = channels * (case["width"] + 1) * e
        states = count * (case["width"] - 1) * channels * e
        if op == "conv_backward":
            return {"bytes": 3 * n * e + 2 * weights + (3 * states if case["state"] else 0), "flops": n * (6 * case["width"] + (8 if case["act"] else 0))}
        given = op == "conv_step" or case["state"]
        return {"bytes": 2 * n * e + weights + states * (2 if given else 1), "flops": n * (2 * case["width"] + (4 if case["act"] else 0))}
    s, groups = case["states"], case["groups"]
    rates = 4 * channels * (s + 2)
    states = 4 * count * channels * s
    if op == "scan_backward":
        wide = n * e * (7 if case["gate"] else 5)
        return {"bytes": wide + tokens * groups * s * e * 4 + 2 * rates + (3 * states if case["state"] else 0), "flops": 20 * n * s}
    given = op == "scan_step" or case["state"]
    return {"bytes": n * e * (4 if case["gate"] else 3) + tokens * groups * s * e * 2 + rates + states * (2 if given else 1), "flops": 7 * n * s}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _starts(case, state):
    """For every token of the flattened ones: the first of its sequence, and the sequence."""
    total = case["tokens"] * case["batch"]
    t = torch.arange(total, device="cuda")
    if state["offsets"] is None:
        seq = t // case["tokens"]
        return t, seq * case["tokens"], seq
    seq = (t[:, None] >= state["offsets"][None, 1:]).sum(1)
    return t, state["offsets"][seq], seq


def _exact_conv(case, state):
    """The inputs `back` tokens in front of every token, by `back`, those of the state among them; the sums; both derivatives."""
    width, channels = case["width"], case["channels"]
    x = state["x"].double().reshape(-1, channels)
    t, first, seq = _starts(case, state)
    taps = []
    for back in range(width):
        at = t - back
        v = x[at.clamp(min=0)]
        if state["s"] is not None:
            front = state["s"].double()[seq, (width - 1 + at - first).clamp(0, width - 2)]
        else:
            front = torch.zeros_like(v)
        taps.append(torch.where((at >= first)[:, None], v, front))
    w = state["weight"].double()
    s = state["bias"].double().expand(t.numel(), -1)
    for back in range(width):
        s = s + taps[back] * w[:, width - 1 - back]
    return x, t, first, seq, taps, w, s


def _ends(case, state):
    if state["offsets"] is None:
        return [(b * case["tokens"], (b + 1) * case["tokens"]) for b in range(case["batch"])]
    o = state["offsets"].tolist()
    return list(zip(o[:-1], o[1:]))


def _exact_conv_forward(case, state):
    x, *_, s = _exact_conv(case, state)
    y = s / (1.0 + torch.exp(-s)) if case["act"] else s
    last = []
    for n, (first, end) in enumerate(_ends(case, state)):
        front = state["s"][n].double() if state["s"] is not None else x.new_zeros(case["width"] - 1, case["channels"])
        last.append(torch.cat([front, x[first:end]])[end - first:])
    return y.reshape(state["x"].shape), torch.stack(last)


def _exact_conv_backward(case, state):
    x, t, first, seq, taps, w, s = _exact_conv(case, state)
    width = case["width"]
    ds = state["dout"].double().reshape(x.shape)
    if case["act"]:
        e = torch.exp(-s)
        ds = ds * (1.0 + e + s * e) / (1.0 + e) ** 2
    dx = torch.zeros_like(x)
    count = case["seqs"] or case["batch"]
    dstate = torch.zeros(count, width - 1, x.shape[1], device="cuda", dtype=torch.float64)
    for back in range(width):
        part, inside = ds * w[:, width - 1 - back], t - back >= first
        dx.index_add_(0, (t - back)[inside], part[inside])
        dstate.index_put_((seq[~inside], (width - 1 + t - back - first)[~inside]), part[~inside], accumulate=True)
    if state["dfinal"] is not None:
        for n, (top, end) in enumerate(_ends(case, state)):
            for j in range(width - 1):
                at = end - (width - 1) + j
                if at >= top:
                    dx[at] += state["dfinal"][n, j].double()
                else:
                    dstate[n, width - 1 + at - top] += state["dfinal"][n, j].double()
    dw = torch.stack([(ds * taps[width - 1 - j]).sum(0) for j in range(width)], 1)
    got = (dx.reshape(state["x"].shape), dw, ds.sum(0))
    return got if state["s"] is None else (*got, dstate)


def _composed(keep, add):
    """All running results of h -> keep h + add along the first axis, by doubling."""
    reach = 1
    while reach < add.shape[0]:
        add = torch.cat([add[:reach], add[reach:] + keep[reach:] * add[:-reach]])
        keep = torch.cat([keep[:reach], keep[reach:] * keep[:-reach]])
        reach *= 2
    return add


def _slices(case, size):
    """The channels in slices whose arrays of 64-bit states take `size` bytes each, none across two groups."""
    each = case["channels"] // case["groups"]
    most = max(1, size // (8 * case["tokens"] * case["batch"] * case["states"]))
    for g in range(case["groups"]):
        for top in range(g * each, (g + 1) * each, most):
            yield g, slice(top, min(top + most, (g + 1) * each))


def _exact_scan(case, state, backward):
    channels, n, total = case["channels"], case["states"], case["tokens"] * case["batch"]

    def flat(name):
        return state[name].reshape(total, *state[name].shape[-2 if name in "bc" else -1:])

    t, first, seq = _starts(case, state)
    ends = _ends(case, state)
    begins, last_of = t == first, torch.zeros(total, dtype=torch.bool, device="cuda")
    filled = [(i, top, end) for i, (top, end) in enumerate(ends) if end > top]
    last_of[[end - 1 for _, _, end in filled]] = True
    out = {k: torch.zeros(total, channels, device="cuda", dtype=torch.float64) for k in (("dx", "ddt", "dz") if backward else ("y",))}
    if backward:
        out |= {k: torch.zeros(total, case["groups"], n, device="cuda", dtype=torch.float64) for k in ("db", "dc")}
        out |= {k: torch.zeros(channels, device="cuda", dtype=torch.float64) for k in ("dskip", "dbias")}
        out["da"] = torch.zeros(channels, n, device="cuda", dtype=torch.float64)
    state_like = torch.zeros(len(ends), channels, n, device="cuda", dtype=torch.float64)
    given, after = state_like, state_like
    if state["s"] is not None:
        given = state["s"].double()
    if backward and state["dfinal"] is not None:
        after = state["dfinal"].double()
    carried = (after if backward else given).clone()              # what an empty sequence hands on
    for g, part in _slices(case, 1 << 30):
        x = flat("x")[:, part].double()
        raw = flat("dt")[:, part].double() + state["dt_bias"][part].double()
        dt = torch.where(raw > 30.0, raw, torch.log1p(torch.exp(raw.clamp(max=30.0))))
        a = state["a"][part].double()
        b, c = flat("b")[:, g].double()[:, None], flat("c")[:, g].double()[:, None]
        keep = torch.exp(dt[..., None] * a)
        # a sequence's first token takes its state in, and nothing from the token in front of it
        before = given[seq][:, part]
        add = (dt * x)[..., None] * b + torch.where(begins[:, None, None], keep * before, 0.0)
        h = _composed(torch.where(begins[:, None, None], 0.0, keep), add)
        y = (h * c).sum(2) + state["skip"][part].double() * x
        z = flat("gate_in")[:, part].double() if case["gate"] else None
        if not backward:
            out["y"][:, part] = y if z is None else y * z / (1.0 + torch.exp(-z))
            for i, _, end in filled:
                carried[i, part] = h[end - 1]
            continue
        dy = flat("dout")[:, part].double()
        if z is not None:
            e = torch.exp(-z)
            out["dz"][:, part] = dy * y * (1.0 + e + z * e) / (1.0 + e) ** 2
            dy = dy * z / (1.0 + e)
        previous = torch.where(begins[:, None, None], before, torch.cat([h[:1], h[:-1]]))
        del before
        # the gradient of h_t: from the token itself, from the next one, or from the state behind the last
        grad = dy[..., None] * c + torch.where(last_of[:, None, None], after[seq][:, part], 0.0)
        follow = torch.where(last_of[:, None, None], 0.0, torch.cat([keep[1:], keep[:1]]))
        grad = _composed(follow.flip(0), grad.flip(0)).flip(0)
        del follow
        out["dc"][:, g] += (dy[..., None] * h).sum(1)
        out["db"][:, g] += (grad * (dt * x)[..., None]).sum(1)
        through = grad * keep * previous
        gb = (grad * b).sum(2)
        out["dx"][:, part] = gb * dt + dy * state["skip"][part].double()
        ddt = (gb * x + (through * a).sum(2)) / (1.0 + torch.exp(-raw))
        out["ddt"][:, part] = ddt
        out["da"][part] = (through * dt[..., None]).sum(0)
        out["dskip"][part], out["dbias"][part] = (dy * x).sum(0), ddt.sum(0)
        for i, top, _ in filled:
            carried[i, part] = (grad * keep)[top]
    shape = state["x"].shape
    if not backward:
        return out["y"].reshape(shape), carried
    got = (out["dx"].reshape(shape), out["ddt"].reshape(shape), out["da"], out["db"].reshape(state["b"].shape), out["dc"].reshape(state["b"].shape),
           out["dskip"])
    if case["gate"]:
        got += (out["dz"].reshape(shape),)
    got += (out["dbias"],)
    return got if state["s"] is None else (*got, carried)


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        norm = torch.sqrt(sum((g.double() ** 2).sum() for g in state["grads"]))
        factor = min(1.0, state["limit"] / (float(norm) + 1e-6))
        buckets = [torch.zeros(b.shape, dtype=torch.float64, device="cuda") for b in state["buckets"]]
        for g, to in zip(state["grads"], state["clipped"]):
            for b, exact_b in zip(state["buckets"], buckets):
                if b.dtype == g.dtype:
                    exact_b[to.storage_offset():to.storage_offset() + g.numel()] = g.double().flatten() * factor
        return (norm, *buckets)
    if op == "conv":
        return _exact_conv_forward(case, state)
    if op == "conv_backward":
        return _exact_conv_backward(case, state)
    if op == "conv_step":
        s, x = state["s"].double(), state["x"].double()
        y = x * state["weight"][:, -1].double() + state["bias"].double()
        for j in range(case["width"] - 1):
            y = y + s[:, j] * state["weight"][:, j].double()
        return (y / (1.0 + torch.exp(-y)) if case["act"] else y), torch.cat([s[:, 1:], x.unsqueeze(1)], 1)
    if op.startswith("scan") and op != "scan_step":
        return _exact_scan(case, state, op == "scan_backward")
    raw = state["dt"].double() + state["dt_bias"].double()
    dt, x = torch.log1p(torch.exp(raw)), state["x"].double()
    each = case["channels"] // case["groups"]
    group = torch.arange(case["channels"], device="cuda") // each
    h = state["s"].double() * torch.exp(dt.unsqueeze(2) * state["a"].double()) + (dt * x).unsqueeze(2) * state["b"].double()[:, group]
    y = (state["c"].double()[:, group] * h).sum(2) + x * state["skip"].double()
    if case["gate"]:
        z = state["gate_in"].double()
        y = y * z / (1.0 + torch.exp(-z))
    return y, h

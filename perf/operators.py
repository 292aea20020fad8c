"""Linear attention with a decay for each head (prompts, their gradients, single tokens) and the root-mean-square norm with
the residual's addition (its gradient, outputs in 8 bits), as cases that can be timed and compared: each in its plain form,
elementary torch operations in 32 bits, and through the library's calls.

A case is a dict of plain values:

  op        "attention", "attention_backward", "attention_step", "norm", "norm_backward"
  dtype     "bf16", "f16" or (norm) "f32": the type of inputs and outputs; states are binary32
  attention: batch x tokens (or `seqs` packed sequences of `tokens` tokens in all), heads, kv_heads, dk, dv;
            state: whether the sequences go on from given states
  norm:     rows, cols; residual: whether one is added; out: "same", "f8" or "i8"; group: columns per scale (0: the row)
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one long prompt
        {"name": "prompt_32k", "op": "attention", "dtype": "bf16", "seqs": 0, "batch": 1, "tokens": 32768, "heads": 16, "kv_heads": 16,
         "dk": 128, "dv": 128, "state": False},
        # prompts of different lengths packed behind one another, an empty one and one of a single token among them, that go on
        # from earlier parts
        {"name": "prompts_packed", "op": "attention", "dtype": "f16", "seqs": 13, "batch": 1, "tokens": 8191, "heads": 8, "kv_heads": 8,
         "dk": 64, "dv": 128, "state": True},
        # a short question, query heads sharing keys and values
        {"name": "prompt_short", "op": "attention", "dtype": "bf16", "seqs": 0, "batch": 1, "tokens": 173, "heads": 16, "kv_heads": 4,
         "dk": 128, "dv": 128, "state": False},
        # the gradients of one training step's sequences
        {"name": "attn_grad_4x2048", "op": "attention_backward", "dtype": "bf16", "seqs": 0, "batch": 4, "tokens": 2048, "heads": 16,
         "kv_heads": 16, "dk": 128, "dv": 128, "state": False},
        # the same for packed sequences with shared keys and values
        {"name": "attn_grad_packed", "op": "attention_backward", "dtype": "f16", "seqs": 9, "batch": 1, "tokens": 5003, "heads": 8,
         "kv_heads": 4, "dk": 64, "dv": 64, "state": False},
        # one conversation's next token: latency
        {"name": "step_1", "op": "attention_step", "dtype": "bf16", "batch": 1, "heads": 16, "kv_heads": 16, "dk": 128, "dv": 128},
        # the next token of a full batch: the states' bytes
        {"name": "step_256", "op": "attention_step", "dtype": "f16", "batch": 256, "heads": 16, "kv_heads": 16, "dk": 128, "dv": 128},
        # the norm in front of an 8-bit product, while tokens are generated
        {"name": "norm_f8_decode", "op": "norm", "dtype": "bf16", "rows": 8, "cols": 4096, "residual": True, "out": "f8", "group": 0},
        # and for a prompt, with a scale for each 128 columns
        {"name": "norm_f8_prompt", "op": "norm", "dtype": "bf16", "rows": 8191, "cols": 5120, "residual": True, "out": "f8", "group": 128},
        # a training step's
        {"name": "norm_16k", "op": "norm", "dtype": "bf16", "rows": 16384, "cols": 4096, "residual": True, "out": "same", "group": 0},
        # its gradients
        {"name": "norm_grad_16k", "op": "norm_backward", "dtype": "bf16", "rows": 16384, "cols": 4096, "residual": True},
        # rows of an odd length
        {"name": "norm_odd", "op": "norm", "dtype": "f16", "rows": 2999, "cols": 1001, "residual": False, "out": "same", "group": 0},
    ]


def _size(rng, low, high):
    """A size between the two, evenly over its logarithm: a power of two a third of the time, odd otherwise."""
    v = 2.0 ** rng.uniform(math.log2(low), math.log2(high))
    return 1 << round(math.log2(v)) if rng.random() < 0.33 else min(int(v) | 1, high)


def draw(rng):
    op = rng.choice(("attention", "attention", "attention_backward", "attention_backward", "attention_step", "norm", "norm", "norm_backward"))
    if op.startswith("norm"):
        case = {"op": op, "dtype": rng.choice(("bf16", "bf16", "f16", "f32")), "residual": rng.random() < 0.6}
        case["cols"] = rng.choice((1024, 2048, 2560, 4096, 5120, 8192, 16384)) if rng.random() < 0.6 else _size(rng, 64, 16384)
        most = (1 << 26) // (2 if case["dtype"] == "f32" else 1) // case["cols"]
        case["rows"] = _size(rng, 1, min(most, 32768))
        if op == "norm":
            case["out"] = rng.choice(("same", "f8", "f8", "i8"))
            case["group"] = rng.choice((0, 32, 64, 128)) if case["out"] != "same" else 0
        return case
    case = {"op": op, "dtype": rng.choice(("bf16", "f16")), "batch": 1}
    case["dk"], case["dv"] = rng.choice(((64, 64), (128, 128), (128, 128), (64, 128), (96, 96), (256, 256), (32, 40)))
    case["kv_heads"] = rng.choice((1, 2, 3, 4, 8))
    case["heads"] = case["kv_heads"] * rng.choice((1, 1, 2))
    if op == "attention_step":
        case["batch"] = _size(rng, 1, min(256, (1 << 26) // (case["heads"] * case["dk"] * case["dv"])))
        return case
    limit = (1 << 26 if op == "attention" else 1 << 24) // (case["heads"] * max(case["dk"], case["dv"]))
    case["seqs"] = rng.choice((0, 0, 5, 13))
    case["batch"] = 1 if case["seqs"] else rng.choice((1, 2, 4))
    limit = min(limit, 32768 if not case["seqs"] else 8192) // case["batch"]
    case["tokens"] = _size(rng, 1 if not case["seqs"] else 512, limit)
    case["state"] = op == "attention" and rng.random() < 0.4
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


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = _TYPES[case["dtype"]]

    def normal(*shape, spread=1.0, dtype=dtype):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * spread).to(dtype)

    state = dict(case)
    if case["op"].startswith("norm"):
        rows, cols = case["rows"], case["cols"]
        state["weight"] = (1.0 + normal(cols, spread=0.2, dtype=torch.float32)).to(dtype)
        if case["op"] == "norm":
            state["x"] = normal(rows, cols)
            state["r"] = normal(rows, cols, spread=3.0) if case["residual"] else None
            return state
        # what the forward pass has left: the sum in front of the norm and the reciprocal root mean square
        state["total"] = normal(rows, cols, spread=3.0)
        state["rstd"] = torch.rsqrt(state["total"].float().square().mean(1) + 1e-6)
        state["dout"] = normal(rows, cols)
        state["dtotal"] = normal(rows, cols) if case["residual"] else None
        return state
    heads, kv, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
    # heads that look back over 8 tokens to heads that look back over a thousand
    state["decay"] = torch.log1p(-torch.exp2(-torch.linspace(3.0, 10.0, heads, device="cuda")))
    if case["op"] == "attention_step":
        batch = case["batch"]
        state |= {"q": normal(batch, heads, dk), "k": normal(batch, kv, dk), "v": normal(batch, kv, dv)}
        state["s"] = normal(batch, heads, dk, dv, spread=4.0, dtype=torch.float32)
        state["next"] = torch.empty_like(state["s"])       # (a pass can be repeated: the new state stands beside the old one)
        return state
    lead = (case["tokens"],) if case["seqs"] else (case["batch"], case["tokens"])
    state |= {"q": normal(*lead, heads, dk), "k": normal(*lead, kv, dk), "v": normal(*lead, kv, dv)}
    state["offsets"], state["longest"] = None, case["tokens"]
    if case["seqs"]:
        state["offsets"] = _lengths(case, gen)
        state["longest"] = int((state["offsets"][1:] - state["offsets"][:-1]).max())
    count = case["seqs"] or case["batch"]
    state["s"] = normal(count, heads, dk, dv, spread=4.0, dtype=torch.float32) if case["state"] else None
    if case["op"] == "attention_backward":
        state["dout"] = normal(*lead, heads, dv)
    return state


# ------------------------------------------------------------------------------------------------ plain forms
_CHUNK = 128


def _rows(x, state):
    """[sequences, heads, longest, d] in 32 bits, every sequence at the end of its row, zeros in front; heads repeated."""
    x = x.float()
    if state["offsets"] is not None:
        o = state["offsets"]
        at = o[1:, None] - state["longest"] + torch.arange(state["longest"], device=x.device)
        x = torch.where((at >= o[:-1, None])[:, :, None, None], x[at.clamp(min=0)], 0.0)
    return x.repeat_interleave(state["heads"] // x.shape[2], 2).transpose(1, 2)


def _back(x, state, kv_heads, dtype):
    """The inverse of _rows: the sum over repeated heads, packed again, rounded."""
    x = x.transpose(1, 2)
    if kv_heads != x.shape[2]:
        x = x.reshape(x.shape[0], x.shape[1], kv_heads, -1, x.shape[3]).sum(3)
    if state["offsets"] is not None:
        o = state["offsets"]
        at = torch.arange(state["tokens"], device=x.device)
        seq = torch.searchsorted(o[1:], at, right=True)
        x = x[seq, at - o[seq + 1] + state["longest"]]
    return x.to(dtype)


def _running(q, k, v, decay, want_state=True):
    """o_t = q_t S_t with S_t = exp(decay) S_{t-1} + k_t v_t^T along the third axis, and the last S: products within chunks, one
    product with a triangular matrix over the chunks' sums."""
    length = q.shape[2]
    size = min(_CHUNK, length)
    chunks = -(-length // size)
    pad = chunks * size - length
    q, k, v = (torch.nn.functional.pad(x, (0, 0, pad, 0)).reshape(x.shape[0], x.shape[1], chunks, size, x.shape[3]) for x in (q, k, v))
    i = torch.arange(size, device=q.device, dtype=torch.float32)
    a = decay[:, None, None]
    rel = i[:, None] - i[None, :]
    within = torch.where(rel >= 0, torch.exp(a * rel.clamp(min=0)), 0.0)                    # [heads, size, size]
    o = torch.matmul(torch.matmul(q, k.transpose(-1, -2)) * within[None, :, None], v)
    if chunks > 1 or want_state:
        sums = torch.matmul((k * torch.exp(a * (size - 1 - i)[:, None])[None, :, None]).transpose(-1, -2), v)
        c = torch.arange(chunks + 1, device=q.device, dtype=torch.float32)
        rel = c[:, None] - 1 - c[None, :chunks]
        between = torch.where(rel >= 0, torch.exp(a * size * rel.clamp(min=0)), 0.0)        # [heads, chunks + 1, chunks]
        states = torch.matmul(between, sums.flatten(3)).unflatten(3, sums.shape[3:])
        o = o + torch.matmul(q * torch.exp(a * (i + 1)[:, None])[None, :, None], states[:, :, :chunks])
    return o.flatten(2, 3)[:, :, pad:], states[:, :, chunks] if want_state else None


def _plain_attention(state):
    q, k, v, decay = (*(_rows(state[n], state) for n in "qkv"), state["decay"])
    scale = state["dk"] ** -0.5
    o, last = _running(q, k, v, decay)
    if state["s"] is not None:
        t = torch.arange(state["longest"], device=q.device, dtype=torch.float32).expand(q.shape[0], -1)
        length = torch.full((q.shape[0],), float(state["longest"]), device=q.device)
        if state["offsets"] is not None:
            length = (state["offsets"][1:] - state["offsets"][:-1]).float()
            t = (t + length[:, None] - state["longest"]).clamp(min=0)
        o = o + torch.matmul(q * torch.exp(decay[None, :, None] * (t + 1)[:, None])[..., None], state["s"])
        last = last + torch.exp(decay * length[:, None])[..., None, None] * state["s"]
    return _back(o * scale, state, state["heads"], state["q"].dtype), last


def _plain_attention_backward(state):
    q, k, v, do = (_rows(state[n], state) for n in ("q", "k", "v", "dout"))
    decay, scale, kv, dtype = state["decay"], state["dk"] ** -0.5, state["kv_heads"], state["q"].dtype
    dq, _ = _running(do, v, k, decay, False)
    q, k, v, do = (x.flip(2) for x in (q, k, v, do))
    dk, _ = _running(v, do, q, decay, False)
    dv, _ = _running(k, q, do, decay, False)
    return (_back(dq * scale, state, state["heads"], dtype), _back(dk.flip(2) * scale, state, kv, dtype),
            _back(dv.flip(2) * scale, state, kv, dtype))


def _plain_attention_step(state):
    group = state["heads"] // state["kv_heads"]
    q, k, v = state["q"].float(), state["k"].float().repeat_interleave(group, 1), state["v"].float().repeat_interleave(group, 1)
    s = torch.exp(state["decay"])[:, None, None] * state["s"] + k[..., None] * v[..., None, :]
    o = torch.matmul(q[..., None, :], s)[..., 0, :] * state["dk"] ** -0.5
    return o.to(state["q"].dtype), s


def _plain_norm(state):
    x, r = state["x"], state["r"]
    s = x.float() if r is None else x.float() + r.float()
    y = s * torch.rsqrt(s.square().mean(1, keepdim=True) + 1e-6) * state["weight"].float()
    total = () if r is None else (s.to(x.dtype),)
    if state["out"] == "same":
        return (y.to(x.dtype), *total)
    rows, cols = y.shape
    group = state["group"] or cols
    most = 448.0 if state["out"] == "f8" else 127.0
    groups = torch.nn.functional.pad(y, (0, -cols % group)).view(rows, -1, group)
    scale = (groups.abs().amax(2) / most).clamp(min=2.0 ** -126)
    codes = (groups / scale[..., None]).flatten(1)[:, :cols]
    if state["out"] == "f8":
        return (codes.to(torch.float8_e4m3fn), scale, *total)
    return (_values(codes.round().to(torch.int8), scale, group, x.dtype), scale, *total)


def _values(codes, scale, group, dtype):
    """What whole numbers in 8 bits stand for."""
    return (codes.float() * scale.repeat_interleave(group, 1)[:, :codes.shape[1]]).to(dtype)


def _plain_norm_backward(state):
    s, dy, w, rstd = state["total"].float(), state["dout"].float(), state["weight"].float(), state["rstd"][:, None]
    g = dy * w
    dx = rstd * (g - s * rstd * rstd * (g * s).mean(1, keepdim=True))
    if state["dtotal"] is not None:
        dx = dx + state["dtotal"].float()
    return dx.to(state["total"].dtype), (dy * s * rstd).sum(0).to(state["weight"].dtype)


# ------------------------------------------------------------------------------------------------ the library's calls
def _own(state):
    from paper_1811_09736_amd import binding
    op = state["op"]
    if op == "attention":
        return binding.linear_attention(state["q"], state["k"], state["v"], state["decay"], offsets=state["offsets"], state=state["s"],
                                        final_state=True)
    if op == "attention_backward":
        return binding.linear_attention_backward(state["dout"], state["q"], state["k"], state["v"], state["decay"],
                                                 offsets=state["offsets"])[:3]
    if op == "attention_step":
        o = binding.linear_attention_step(state["q"], state["k"], state["v"], state["decay"], state["s"], new_state=state["next"])
        return o, state["next"]
    if op == "norm_backward":
        return binding.rms_norm_backward(state["dout"], state["total"], state["weight"], state["rstd"], dtotal=state["dtotal"])
    if state["out"] == "same":
        y = binding.rms_norm(state["x"], state["weight"], residual=state["r"], eps=1e-6)
        return y if isinstance(y, tuple) else (y,)
    kind = torch.float8_e4m3fn if state["out"] == "f8" else torch.int8
    codes, scale, *total = binding.rms_norm_quantized(state["x"], state["weight"], residual=state["r"], eps=1e-6, dtype=kind,
                                                      group=state["group"])
    if state["out"] == "i8":
        codes = _values(codes, scale, state["group"] or state["cols"], state["x"].dtype)
    return (codes, scale, *total)


_PLAIN = {"attention": _plain_attention, "attention_backward": _plain_attention_backward, "attention_step": _plain_attention_step,
          "norm": _plain_norm, "norm_backward": _plain_norm_backward}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


def work(case):
    """Inputs read once, outputs written once.  Attention by its recurrence: a multiplication and an addition for each entry of
    the state and each product with it."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("norm"):
        n, cols = case["rows"] * case["cols"], case["cols"]
        if case["op"] == "norm_backward":
            return {"bytes": n * e * (4 if case["residual"] else 3) + 4 * case["rows"] + 2 * cols * e, "flops": 9 * n}
        out = n * e if case["out"] == "same" else n + 4 * case["rows"] * (-(-cols // case["group"]) if case["group"] else 1)
        return {"bytes": n * e * (3 if case["residual"] else 1) + out + cols * e, "flops": 5 * n}
    heads, kv, dk, dv = case["heads"], case["kv_heads"], case["dk"], case["dv"]
    if case["op"] == "attention_step":
        n = case["batch"]
        return {"bytes": n * (8 * heads * dk * dv + e * (heads + kv) * (dk + dv)), "flops": 5 * n * heads * dk * dv}
    n = case["tokens"] * case["batch"]
    sequences = case["seqs"] or case["batch"]
    if case["op"] == "attention":
        states = 4 * sequences * heads * dk * dv * (2 if case["state"] else 1)
        return {"bytes": n * e * (heads + kv) * (dk + dv) + states, "flops": 4 * n * heads * dk * dv}
    return {"bytes": n * e * (heads * (2 * dk + dv) + 2 * kv * (dk + dv)), "flops": 10 * n * heads * dk * dv}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _spans(state):
    """(index of the leading axes, length) of every sequence."""
    if state["offsets"] is None:
        return [((b, slice(0, state["tokens"])), state["tokens"]) for b in range(state["batch"])]
    o = state["offsets"].tolist()
    return [((slice(o[s], o[s + 1]),), o[s + 1] - o[s]) for s in range(len(o) - 1)]


def _weights(decay, top, end, device):
    """decay^(i - j) for rows i = top .. end - 1 and columns j < end; 0 where j > i."""
    i = torch.arange(top, end, device=device, dtype=torch.float64)[:, None]
    j = torch.arange(end, device=device, dtype=torch.float64)[None, :]
    return torch.where(j <= i, torch.exp(decay * (i - j).clamp(min=0)), 0.0)


def _exact_attention(state):
    q, k, v, decay = (state[n].double() for n in ("q", "k", "v", "decay"))
    scale, group = state["dk"] ** -0.5, state["heads"] // state["kv_heads"]
    o = torch.zeros(*q.shape[:-1], state["dv"], device=q.device, dtype=torch.float64)
    last = torch.zeros(len(_spans(state)), state["heads"], state["dk"], state["dv"], device=q.device, dtype=torch.float64)
    for n, (at, length) in enumerate(_spans(state)):
        for h in range(state["heads"]):
            qh, kh, vh, a = q[at][:, h], k[at][:, h // group], v[at][:, h // group], decay[h]
            s = state["s"][n, h].double() if state["s"] is not None else torch.zeros_like(last[n, h])
            for top in range(0, length, 2048):
                end = min(top + 2048, length)
                o[at][top:end, h] = scale * ((qh[top:end] @ kh[:end].T * _weights(a, top, end, q.device)) @ vh[:end])
            t = torch.arange(length, device=q.device, dtype=torch.float64)
            o[at][:, h] += scale * torch.exp(a * (t + 1))[:, None] * (qh @ s)
            last[n, h] = (kh * torch.exp(a * (length - 1 - t))[:, None]).T @ vh + torch.exp(a * length) * s
    return o, last


def _exact_attention_backward(state):
    q, k, v, do, decay = (state[n].double() for n in ("q", "k", "v", "dout", "decay"))
    scale, group = state["dk"] ** -0.5, state["heads"] // state["kv_heads"]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for at, length in _spans(state):
        for h in range(state["heads"]):
            g = h // group
            qh, kh, vh, doh = q[at][:, h], k[at][:, g], v[at][:, g], do[at][:, h]
            for top in range(0, length, 2048):
                end = min(top + 2048, length)
                w = scale * _weights(decay[h], top, end, q.device)
                score, grad = w * (qh[top:end] @ kh[:end].T), w * (doh[top:end] @ vh[:end].T)
                dq[at][top:end, h] += grad @ kh[:end]
                dk[at][:end, g] += grad.T @ qh[top:end]
                dv[at][:end, g] += score.T @ doh[top:end]
    return dq, dk, dv


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "attention":
        return _exact_attention(state)
    if op == "attention_backward":
        return _exact_attention_backward(state)
    if op == "attention_step":
        group = case["heads"] // case["kv_heads"]
        q, k, v = state["q"].double(), state["k"].double().repeat_interleave(group, 1), state["v"].double().repeat_interleave(group, 1)
        s = state["s"].double() * state["decay"].double().exp()[None, :, None, None] + k.unsqueeze(3) * v.unsqueeze(2)
        return (q.unsqueeze(3) * s).sum(2) / math.sqrt(case["dk"]), s
    w = state["weight"].double()
    if op == "norm_backward":
        s, dy, r = state["total"].double(), state["dout"].double(), state["rstd"].double().unsqueeze(1)
        unit = s * r
        dx = r * (dy * w) - r * unit * (dy * w * unit).sum(1, keepdim=True) / case["cols"]
        return (dx if state["dtotal"] is None else dx + state["dtotal"].double()), (dy * unit).sum(0)
    s = state["x"].double() + (state["r"].double() if case["residual"] else 0.0)
    y = w * s / torch.sqrt((s * s).sum(1, keepdim=True) / case["cols"] + 1e-6)
    total = (s,) if case["residual"] else ()
    if case["out"] == "same":
        return (y, *total)
    group = case["group"] or case["cols"]
    scales = torch.stack([part.abs().amax(1) for part in y.split(group, 1)], 1) / (448.0 if case["out"] == "f8" else 127.0)
    # the values that the codes stand for before they are rounded (bytes of a floating type: in units of the scale)
    return (y / scales.repeat_interleave(group, 1)[:, :case["cols"]] if case["out"] == "f8" else y, scales, *total)

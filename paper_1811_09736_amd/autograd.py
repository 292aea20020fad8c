"""Linear attention with decay, the root-mean-square norm, the short causal convolution and the selective scan as differentiable functions: binding's calls
and their gradients, nothing else (gradients of the gradients are refused)."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, scale, offsets, state):
        out, last = binding.linear_attention(q, k, v, log_decay, scale=scale, offsets=offsets, state=state, final_state=True)
        ctx.save_for_backward(q, k, v, log_decay, offsets, state)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        q, k, v, log_decay, offsets, state = ctx.saved_tensors
        if dout is None:
            dout = torch.zeros(*q.shape[:-1], v.shape[-1], dtype=q.dtype, device=q.device)
        if dout.stride(-1) != 1:
            dout = dout.contiguous()
        dlast = None if dlast is None else dlast.contiguous()
        dq, dk, dv, dstate = binding.linear_attention_backward(dout, q, k, v, log_decay, scale=ctx.scale, offsets=offsets, state=state, dfinal=dlast)
        return dq, dk, dv, None, None, None, dstate


def linear_attention(q, k, v, log_decay, scale=None, offsets=None, state=None):
    """binding.linear_attention with gradients for q, k, v and state: (out, the states behind the last tokens).  log_decay is a constant: one that
    requires a gradient, and would never get it, is refused."""
    if log_decay.requires_grad and torch.is_grad_enabled():
        raise ValueError("log_decay must not require a gradient: the decays are constants of the model here (pass log_decay.detach())")
    return _LinearAttention.apply(q, k, v, log_decay, scale, offsets, state)


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, residual, eps):
        if residual is None:
            out, rstd = binding.rms_norm(x, weight, eps=eps, rstd=True)
            total = x
        else:
            out, total, rstd = binding.rms_norm(x, weight, residual=residual, eps=eps, rstd=True)
        ctx.save_for_backward(total, weight, rstd)
        ctx.added = residual is not None
        ctx.set_materialize_grads(False)
        return (out, total) if ctx.added else out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dtotal=None):
        total, weight, rstd = ctx.saved_tensors
        dout = torch.zeros_like(total) if dout is None else dout.contiguous()
        dx, dweight = binding.rms_norm_backward(dout, total, weight, rstd, dtotal=None if dtotal is None else dtotal.contiguous())
        return dx, dweight, dx if ctx.added else None, None


def rms_norm(x, weight, residual=None, eps=1e-6):
    """binding.rms_norm with gradients for x, weight and residual: the norm, with a residual (the norm, x + residual)."""
    return _RmsNorm.apply(x, weight, residual, eps)


def _whole(grad, like):
    """The gradient of an output of `like`'s shape: zeros where the output was not used, its last dimension contiguous."""
    if grad is None:
        return torch.zeros(like.shape, dtype=like.dtype, device=like.device)
    return grad if grad.stride(-1) == 1 else grad.contiguous()


class _CausalConv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, activation, offsets, state):
        ctx.save_for_backward(x, weight, bias, offsets, state)
        ctx.activation = activation
        ctx.set_materialize_grads(False)
        return binding.causal_conv(x, weight, bias=bias, activation=activation, offsets=offsets, state=state, final_state=True)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        x, weight, bias, offsets, state = ctx.saved_tensors
        dx, dweight, dbias, dstate = binding.causal_conv_backward(_whole(dout, x), x, weight, bias=bias, activation=ctx.activation, offsets=offsets, state=state,
                                                                  dfinal=None if dlast is None else dlast.contiguous())
        return dx, dweight, dbias, None, None, dstate


def causal_conv(x, weight, bias=None, activation="silu", offsets=None, state=None):
    """binding.causal_conv with gradients for x, weight, bias and state: (out, the last width - 1 inputs of every sequence)."""
    return _CausalConv.apply(x, weight, bias, activation, offsets, state)


class _SelectiveScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, a, b, c, skip, gate, dt_bias, softplus, offsets, state):
        ctx.save_for_backward(x, dt, a, b, c, skip, gate, dt_bias, offsets, state)
        ctx.softplus = softplus
        ctx.set_materialize_grads(False)
        return binding.selective_scan(x, dt, a, b, c, skip=skip, gate=gate, dt_bias=dt_bias, softplus=softplus, offsets=offsets, state=state, final_state=True)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout, dlast):
        x, dt, a, b, c, skip, gate, dt_bias, offsets, state = ctx.saved_tensors
        dx, ddt, da, db, dc, dskip, dgate, dbias, dstate = binding.selective_scan_backward(
            _whole(dout, x), x, dt, a, b, c, skip=skip, gate=gate, dt_bias=dt_bias, softplus=ctx.softplus, offsets=offsets, state=state,
            dfinal=None if dlast is None else dlast.contiguous())
        return dx, ddt, da, db, dc, dskip, dgate, dbias, None, None, dstate


def selective_scan(x, dt, a, b, c, skip=None, gate=None, dt_bias=None, softplus=True, offsets=None, state=None):
    """binding.selective_scan with gradients for x, dt, a, b, c, skip, gate, dt_bias and state: (out, the states behind the last tokens)."""
    return _SelectiveScan.apply(x, dt, a, b, c, skip, gate, dt_bias, softplus, offsets, state)

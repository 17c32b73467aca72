"""Autograd functions over the layers' entry points: dropout, root-mean-square norms and gated blocks of all replicas at once.

`LASGD` in torch_api.py offers them as methods.  Activations are [K, ..., columns], replica by replica; weights are named once and stand for
every replica's own.  The backward passes add the weights' gradients to the bound buffers themselves, so these never travel through autograd: a weight's
hooks do not run, and `torch.autograd.grad` does not return them.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import torch
from torch.autograd.function import once_differentiable

from . import binding as B

ACTIVATIONS = {"silu": B.SILU, "gelu": B.GELU, "gelu_tanh": B.GELU_TANH, "relu": B.RELU}


class Rows:
    """How a call sees an activation [K, ..., columns]: as [K, rows, columns], without a copy where its strides allow it."""

    def __init__(self, opt, shape, counts: Optional[Sequence[int]]):
        K = len(opt.replicas)
        if len(shape) < 2 or shape[0] != K:
            raise ValueError(f"an activation of {K} replicas is [{K}, ..., columns], this one is {tuple(shape)}")
        most = math.prod(shape[1:-1])
        if counts is None:
            self.counts = [most] * K
        else:
            self.counts = [int(n) for n in counts]
            if len(self.counts) != K or any(n < 0 or n > most for n in self.counts):
                raise ValueError(f"rows: {K} counts of at most {most}, got {self.counts}")
        self.K, self.most, self.whole = K, most, counts is None

    def view(self, opt, t: torch.Tensor, name: str) -> torch.Tensor:
        if t.dtype != opt.dtype or t.device != opt.device:
            raise ValueError(f"{name} is {t.dtype} on {t.device}, the replicas are {opt.dtype} on {opt.device}")
        t = t.reshape(self.K, self.most, t.shape[-1])
        return t if t.stride(2) == 1 or t.shape[2] == 1 else t.contiguous()

    def new(self, like: torch.Tensor, cols: int, dtype=None) -> torch.Tensor:
        """[K, rows, cols]; rows behind a replica's last hold zeros."""
        make = torch.empty if self.whole else torch.zeros
        return make(self.K, self.most, cols, dtype=dtype or like.dtype, device=like.device)


def _at(t: Optional[torch.Tensor]):
    return None if t is None else (t.data_ptr(), t.stride(0), t.stride(1))


def _stream(opt) -> int:
    return torch.cuda.current_stream(opt.device).cuda_stream


def _workspace(opt, nbytes: int) -> Optional[torch.Tensor]:
    return torch.empty(nbytes, dtype=torch.uint8, device=opt.device) if nbytes else None


def _anchor(opt) -> Optional[torch.Tensor]:
    """Something that wants a gradient, so that a call on inputs that want none has a backward pass for its weights.  A new one for each call: a leaf
    that lives on would tie recorded passes to the stream of the first."""
    return torch.empty(0, device=opt.device, requires_grad=True) if torch.is_grad_enabled() else None


class Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, opt, rows, x, residual, drop):
        v, cols = rows.view(opt, x, "x"), x.shape[-1]
        r = None if residual is None else rows.view(opt, residual, "residual")
        y = rows.new(v, cols)
        with torch.cuda.device(opt.device):
            opt.ctx.dropout(rows.counts, cols, _at(v), _at(y), residual=_at(r), stream=_stream(opt), **drop)
        ctx.opt, ctx.rows, ctx.drop = opt, rows, drop
        return y.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        opt, rows, dx = ctx.opt, ctx.rows, None
        if ctx.needs_input_grad[2]:
            v = rows.view(opt, dy, "the gradient")
            dx = rows.new(v, dy.shape[-1])
            with torch.cuda.device(opt.device):
                opt.ctx.dropout(rows.counts, dy.shape[-1], _at(v), _at(dx), stream=_stream(opt), **ctx.drop)
            dx = dx.view(dy.shape)
        return None, None, dx, _rows_of(rows, dy) if ctx.needs_input_grad[3] else None, None


def _rows_of(rows, g):
    """A gradient that passes through: zeros behind a replica's last row, where the output holds none of the input."""
    if rows.whole:
        return g
    at = torch.arange(rows.most, device=g.device)
    there = torch.stack([at < n for n in rows.counts])
    return torch.where(there[:, :, None], g.reshape(rows.K, rows.most, g.shape[-1]), 0).view(g.shape)


class RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, opt, rows, gain, x, residual, anchor, eps, drop, want_sum):
        v, cols = rows.view(opt, x, "x"), x.shape[-1]
        r = None if residual is None else rows.view(opt, residual, "residual")
        y = rows.new(v, cols)
        h = rows.new(v, cols) if r is not None or drop["p"] > 0.0 else None
        with torch.cuda.device(opt.device):
            opt.ctx.rms_norm(gain, rows.counts, _at(v), _at(y), residual=_at(r), sum=_at(h), eps=eps, stream=_stream(opt), **drop)
        ctx.opt, ctx.rows, ctx.gain, ctx.eps, ctx.drop, ctx.shape = opt, rows, gain, eps, drop, x.shape
        ctx.save_for_backward(v if h is None else h)
        ctx.set_materialize_grads(False)
        if not want_sum:
            return y.view(x.shape)
        return y.view(x.shape), h.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dsum=None):
        opt, rows, gain = ctx.opt, ctx.rows, ctx.gain
        h, = ctx.saved_tensors
        if dy is None and dsum is None:
            return (None,) * 9
        dy = torch.zeros(ctx.shape, dtype=h.dtype, device=h.device) if dy is None else dy
        cols = ctx.shape[-1]
        v, s = rows.view(opt, dy, "the gradient"), None if dsum is None else rows.view(opt, dsum, "the gradient of the sum")
        dropped = ctx.drop["p"] > 0.0
        dres = rows.new(h, cols) if ctx.needs_input_grad[4] or (ctx.needs_input_grad[3] and not dropped) else None
        dx = rows.new(h, cols) if ctx.needs_input_grad[3] and dropped else None
        opt._check_weights(gain)
        grads = opt._grads_to_add_to(gain)
        with torch.cuda.device(opt.device):
            work = _workspace(opt, opt.ctx.rms_norm_backward_bytes(gain, rows.counts))
            opt.ctx.rms_norm_backward(gain, rows.counts, _at(h), _at(v), _at(dx), dsum=_at(s), dresidual=_at(dres), eps=ctx.eps, accumulate=True,
                                      workspace=None if work is None else work.data_ptr(), workspace_bytes=0 if work is None else work.numel(),
                                      stream=_stream(opt), **ctx.drop)
        torch.autograd.graph.increment_version(grads)
        dres = None if dres is None else dres.view(ctx.shape)
        dx = dx.view(ctx.shape) if dropped and dx is not None else dres
        return None, None, None, dx if ctx.needs_input_grad[3] else None, dres if ctx.needs_input_grad[4] else None, None, None, None, None


class Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, opt, rows, gate, up, x, anchor, activation):
        v, cols = rows.view(opt, x, "x"), x.shape[-1]
        wide = opt.ctx.numels[gate] // (cols * (2 if gate == up else 1))
        a = rows.new(v, wide)
        keep = anchor is not None
        g, u = (torch.empty_like(a), torch.empty_like(a)) if keep else (None, None)
        with torch.cuda.device(opt.device):
            opt.ctx.gated(gate, up, rows.counts, cols, _at(v), _at(a), g=_at(g), u=_at(u), activation=activation, stream=_stream(opt))
        if keep:
            ctx.save_for_backward(v, g, u)
        ctx.opt, ctx.rows, ctx.gate, ctx.up, ctx.activation, ctx.shape = opt, rows, gate, up, activation, x.shape
        return a.view(*x.shape[:-1], wide)

    @staticmethod
    @once_differentiable
    def backward(ctx, da):
        opt, rows, gate, up = ctx.opt, ctx.rows, ctx.gate, ctx.up
        x, g, u = ctx.saved_tensors
        cols = ctx.shape[-1]
        v = rows.view(opt, da, "the gradient")
        dx = rows.new(x, cols) if ctx.needs_input_grad[4] else None
        opt._check_weights(*{gate, up})
        grads = opt._grads_to_add_to(gate) + ([] if gate == up else opt._grads_to_add_to(up))
        with torch.cuda.device(opt.device):
            work = _workspace(opt, opt.ctx.gated_backward_bytes(gate, up, rows.counts, cols))
            opt.ctx.gated_backward(gate, up, rows.counts, cols, _at(x), _at(g), _at(u), _at(v), _at(dx), activation=ctx.activation, accumulate=True,
                                   workspace=None if work is None else work.data_ptr(), workspace_bytes=0 if work is None else work.numel(),
                                   stream=_stream(opt))
        torch.autograd.graph.increment_version(grads)
        return None, None, None, None, None if dx is None else dx.view(ctx.shape), None, None

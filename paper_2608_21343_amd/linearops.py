"""The output layer and its cross entropy over torch tensors, without the logits.

Marshalling only, as in ``rowops``: all work runs in libtbias.so
(tb_linear_xent and its gradient), in pieces of the vocabulary. ``linear_xent``
is a torch.autograd function whose backward pass makes the logits again from the
rows' log-sum-exp; ``linear_xent_step`` gives loss and gradients in one call.
Gradients are not themselves differentiable: a second derivative raises an error.
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import capi
from .rowops import _constant, _once


class LinearLoss(NamedTuple):
    """Per row of the features [..., width]: weighted loss and log-sum-exp [...]."""

    loss: torch.Tensor
    lse: torch.Tensor


def _even(t: torch.Tensor, name: str) -> torch.Tensor:
    """The rows of a matrix, copied where they are not evenly spaced."""
    try:
        capi._matrix(t, name)
        return t
    except ValueError:
        return t.contiguous()


def _args(x, w, target, bias, weight):
    lead = x.shape[:-1]
    if target.shape != lead:
        raise ValueError("target must be [...] for x [..., width]")
    if weight is not None and weight.shape != lead:
        raise ValueError("weight must be [...] for x [..., width]")
    return (_even(x, "x"), _even(w, "w"), target.contiguous(),
            None if bias is None else bias.contiguous(),
            None if weight is None else weight.contiguous())


def _mark(node) -> None:
    """A backward pass that is captured while a graph of an eager pass over the same
    leaves is alive would wait, inside the capture, for the stream of that pass
    (torch gives a leaf's accumulation the stream of its first use), and end the
    process when the capture ends: such a call is refused here. The marks are on
    the accumulations that follow ``node``, which live as long as a graph of theirs."""
    capturing = torch.cuda.is_current_stream_capturing()
    for leaf, _ in node.next_functions:
        if leaf is not None and leaf.name() == "torch::autograd::AccumulateGrad":
            marks = leaf.metadata
            if not capturing:
                marks["tbias_eager"] = True
            elif marks.get("tbias_eager"):
                raise RuntimeError("a graph of an eager pass over this layer is alive: drop its "
                                   "losses before the capture")


class _LinearXent(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, target, bias, weight):
        x, w, target, bias, weight = _args(x, w, target, bias, weight)
        loss = torch.empty(target.shape, dtype=torch.float32, device=x.device)
        lse, low = torch.empty_like(loss), torch.empty_like(loss)
        capi.tb_linear_xent(x, w, target, loss, lse, bias=bias, weight=weight, out_low=low)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x, w, target, bias, weight, lse, low)
        return loss, lse

    @staticmethod
    def backward(ctx, d_loss, d_lse):
        x, w, target, bias, weight, lse, low = ctx.saved_tensors
        need_x, need_w, _, need_b, _ = ctx.needs_input_grad
        dx = x.new_empty(x.shape) if need_x else None
        dw = w.new_empty(w.shape) if need_w else None
        db = torch.empty_like(bias) if need_b else None
        if d_loss is None:
            d_loss = torch.zeros_like(lse)
        elif any(d_loss.stride()):  # (a sum's gradient is one value, expanded)
            d_loss = d_loss.contiguous()
        capi.tb_linear_xent_grad(x, w, target, lse, d_loss,
                                 None if d_lse is None else d_lse.contiguous(), dx, dw, db,
                                 bias=bias, weight=weight, lse_low=low)
        return tuple(None if g is None else _once(g) for g in (dx, dw, None, db, None))


def linear_xent(x: torch.Tensor, w: torch.Tensor, target: torch.Tensor,
                bias: Optional[torch.Tensor] = None,
                weight: Optional[torch.Tensor] = None) -> LinearLoss:
    """Cross entropy of the logits ``x @ w.T + bias`` against ``target`` (int32
    [...], -1: none) and their log-sum-exp, per row of ``x`` [..., width]; ``w``
    [V+1, width] and ``bias`` [V+1] have the type of ``x`` (float32 or bfloat16).
    ``weight`` [...] multiplies the losses; rows of weight 0 or without a target
    are left out (loss and lse 0). Differentiable with respect to x, w and bias;
    a weight that requires a gradient is refused, and so is a call under graph
    capture while the graph of an eager call with the same leaves is alive."""
    _constant(weight, "weight")
    out = _LinearXent.apply(x, w, target, bias, weight)
    if out[0].requires_grad:
        _mark(out[0].grad_fn)
    return LinearLoss(*out)


def linear_xent_step(x: torch.Tensor, w: torch.Tensor, target: torch.Tensor,
                     bias: Optional[torch.Tensor] = None,
                     weight: Optional[torch.Tensor] = None):
    """(loss [...], and the gradients of its sum with respect to x, w and bias:
    None without one) in one call."""
    x, w, target, bias, weight = _args(x, w, target, bias, weight)
    loss = torch.empty(target.shape, dtype=torch.float32, device=x.device)
    dx, dw = x.new_empty(x.shape), w.new_empty(w.shape)
    db = None if bias is None else torch.empty_like(bias)
    capi.tb_linear_xent(x, w, target, loss, None, dx, dw, db, bias=bias, weight=weight)
    return loss, dx, dw, db

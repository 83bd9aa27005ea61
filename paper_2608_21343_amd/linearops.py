"""The output layer and its cross entropy over torch tensors, without the logits.

Marshalling only, as in ``rowops``: all work runs in libtbias.so
(tb_linear_xent and its gradient), in pieces of the vocabulary. ``linear_xent``
is a torch.autograd function whose backward pass makes the logits again from the
rows' log-sum-exp; ``linear_xent_step`` gives loss and gradients in one call.
Gradients are not themselves differentiable: a second derivative raises an error.
"""

from __future__ import annotations

import weakref
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


class _Eager:
    """An eager call whose graph is alive: it lies in the metadata of the call's node
    and names the nodes that follow."""

    def __init__(self, node):
        self.inputs = [n for n, _ in node.next_functions if n is not None]


_eager = weakref.WeakSet()


def _leaves(nodes) -> set:
    """The accumulations that a backward pass through these nodes reaches."""
    seen, todo = set(), list(nodes)
    while todo:
        node = todo.pop()
        if node not in seen:
            seen.add(node)
            todo += [n for n, _ in node.next_functions if n is not None]
    return {n for n in seen if n.name() == "torch::autograd::AccumulateGrad"}


def _mark(node) -> None:
    """A backward pass that is captured while a graph of an eager pass over the same
    leaves is alive would wait, inside the capture, for the stream of that pass
    (torch gives a leaf's accumulation the stream of its first use). Where that is
    the default stream, which no capture may wait for, the process would end with the
    capture: such a call is refused here, however far behind the call the leaves
    are. Only a call that is captured looks that far."""
    if not torch.cuda.is_current_stream_capturing():
        if not (torch.cuda.is_initialized() and capi._stream(None)):  # (0: the default one)
            call = node.metadata["tbias_eager"] = _Eager(node)
            _eager.add(call)
        return
    mine = _leaves([node])
    for call in list(_eager):
        if not mine.isdisjoint(_leaves(call.inputs)):
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
    capture while the graph of an eager call on the default stream is alive that
    shares a leaf with it (one on another stream, as a capture is warmed up on, may be)."""
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

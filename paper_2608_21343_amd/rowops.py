"""Row operators over torch tensors: confidences of decoded tokens, and losses
for training the joint network whose logits the decoders read.

Marshalling only, as in ``decoder``: buffers come from torch, all work runs in
libtbias.so (tb_token_logprobs, tb_distill and their gradients), and the losses
are torch.autograd functions whose backward passes are those of the library. A
backward pass reads the logits again instead of keeping the probabilities: one
read and one write of their size, and no memory between the passes. Gradients
are not themselves differentiable: a second derivative raises an error.
"""

from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import capi


class TokenScores(NamedTuple):
    """Per row of the logits [..., V+1]: log probabilities [..., n] of the given
    tokens, log-sum-exp and entropy [...], the best alternatives' ids and log
    probabilities [..., m] (ids -1 where a row has fewer)."""

    logprob: torch.Tensor
    lse: torch.Tensor
    entropy: torch.Tensor
    alt: torch.Tensor
    alt_logprob: torch.Tensor


def _even(logits: torch.Tensor) -> torch.Tensor:
    """The logits, copied where their rows are not evenly spaced."""
    try:
        capi._rows(logits)
        return logits
    except ValueError:
        return logits.contiguous()


class _Once(torch.autograd.Function):
    """Passes a gradient on whose own derivative is asked for and not there."""

    @staticmethod
    def forward(ctx, grad):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the row operators have no second derivative: their gradient with "
                           "respect to the logits is a constant to autograd")


def _once(grad: torch.Tensor) -> torch.Tensor:
    """The result of a backward pass. Where a graph of that pass is built
    (create_graph), differentiating it again raises an error: torch's
    once_differentiable does not where only the logits require a gradient."""
    return _Once.apply(grad.requires_grad_()) if torch.is_grad_enabled() else grad


class _TokenScores(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, n_alt, temperature):
        z = _even(logits.detach())
        lead = z.shape[:-1]
        f32 = dict(dtype=torch.float32, device=z.device)
        lp = torch.empty(tokens.shape, **f32)
        lse, ent = torch.empty(lead, **f32), torch.empty(lead, **f32)
        alt = torch.empty((*lead, n_alt), dtype=torch.int32, device=z.device)
        alt_lp = torch.empty((*lead, n_alt), **f32)
        J = tokens.shape[-1]
        capi.tb_token_logprobs(z, tokens if J else None, lp if J else None, lse, ent,
                               alt if n_alt else None, alt_lp if n_alt else None,
                               temperature=temperature)
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(z, tokens, alt)
        ctx.temperature = temperature
        ctx.mark_non_differentiable(alt)
        return lp, lse, ent, alt, alt_lp

    @staticmethod
    def backward(ctx, d_lp, d_lse, d_ent, _, d_alt):
        z, tokens, alt = ctx.saved_tensors
        # the alternatives are tokens like the given ones
        places = [(t, d) for t, d in ((tokens, d_lp), (alt, d_alt))
                  if d is not None and t.shape[-1] > 0]
        tok = d_tok = None
        if places:
            tok = torch.cat([t for t, _ in places], -1) if len(places) > 1 else places[0][0]
            d_tok = torch.cat([d for _, d in places], -1) if len(places) > 1 else places[0][1]

        def row(d):
            return None if d is None else d.contiguous()

        wide = 0 if tok is None else tok.shape[-1]
        if wide <= capi.TB_MAX_LIST:
            grad = torch.empty(z.shape, dtype=z.dtype, device=z.device)
            capi.tb_token_logprobs_grad(z, tok, row(d_tok), grad, row(d_lse), row(d_ent),
                                        temperature=ctx.temperature)
        else:
            # two lists that make no single one: a gradient each in float32, so that
            # bfloat16 rounds their sum once
            (t0, d0), (t1, d1) = places
            z32 = z.float()
            grad, more = torch.empty_like(z32), z32 if z32 is not z else torch.empty_like(z32)
            capi.tb_token_logprobs_grad(z32, t0, row(d0), grad, row(d_lse), row(d_ent),
                                        temperature=ctx.temperature)
            capi.tb_token_logprobs_grad(z32, t1, row(d1), more, temperature=ctx.temperature)
            grad = grad.add_(more).to(z.dtype)
        return _once(grad), None, None, None


def token_scores(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, n_alt: int = 0,
                 temperature: float = 1.0) -> TokenScores:
    """Log probabilities of ``tokens`` (int32 [..., n], or [...] for one token a
    row; -1: none), log-sum-exp, entropy and the ``n_alt`` best alternatives of
    every row of ``logits`` ([..., V+1] float32 or bfloat16 on the device).
    Differentiable with respect to the logits in every floating output."""
    lead = logits.shape[:-1]
    single = tokens is not None and tokens.shape == lead
    if tokens is None:
        tok = torch.empty((*lead, 0), dtype=torch.int32, device=logits.device)
    else:
        tok = tokens.unsqueeze(-1) if single else tokens
        if tok.shape[:-1] != lead:
            raise ValueError("tokens must be [...] or [..., n] for logits [..., V+1]")
        tok = tok.contiguous()
    lp, lse, ent, alt, alt_lp = _TokenScores.apply(logits, tok, int(n_alt), float(temperature))
    return TokenScores(lp.squeeze(-1) if single else lp, lse, ent, alt, alt_lp)


def _constant(t: Optional[torch.Tensor], name: str) -> None:
    if t is not None and t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which this loss does not give: detach it")


def _teacher(logits: torch.Tensor, tok: torch.Tensor, score: torch.Tensor,
             weight: Optional[torch.Tensor]):
    """The teacher's tensors, contiguous; their rows have to be the logits' rows."""
    lead = logits.shape[:-1]
    if tok.dim() != len(lead) + 1 or tok.shape[:-1] != lead:
        raise ValueError("teacher_tok must be [..., k] for logits [..., V+1]")
    if score.shape != tok.shape:
        raise ValueError("teacher_score must have teacher_tok's shape")
    if weight is not None and weight.shape != lead:
        raise ValueError("weight must be [...] for logits [..., V+1]")
    return tok.contiguous(), score.contiguous(), None if weight is None else weight.contiguous()


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tok, score, weight, temperature, tail):
        z = _even(logits.detach())
        loss = torch.empty(z.shape[:-1], dtype=torch.float32, device=z.device)
        capi.tb_distill(z, tok, score, loss, weight=weight, temperature=temperature, tail=tail)
        ctx.save_for_backward(z, tok, score, weight)
        ctx.how = (temperature, tail)
        return loss

    @staticmethod
    def backward(ctx, d_loss):
        z, tok, score, weight = ctx.saved_tensors
        temperature, tail = ctx.how
        w = (d_loss if weight is None else d_loss * weight).contiguous()
        grad = torch.empty(z.shape, dtype=z.dtype, device=z.device)
        capi.tb_distill(z, tok, score, None, grad, weight=w, temperature=temperature, tail=tail)
        return _once(grad), None, None, None, None, None


def distill_loss(logits: torch.Tensor, teacher_tok: torch.Tensor, teacher_score: torch.Tensor,
                 temperature: float = 1.0, tail: bool = False,
                 weight: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Loss [...] of every row of a student's ``logits`` [..., V+1] against a
    teacher's list: tokens int32 [..., k] (-1: unused) and scores float32
    [..., k]. Without the tail the teacher is the softmax of score /
    temperature over its list; with it the scores are log probabilities (a
    teacher's TokenScores at the same temperature) and all other tokens count as
    one event. ``weight`` [...] multiplies the rows. Differentiable with respect
    to the logits alone: scores and weights that require a gradient are refused.
    distill_step gives loss and gradient in one pass."""
    _constant(teacher_score, "teacher_score")
    _constant(weight, "weight")
    return _Distill.apply(logits, *_teacher(logits, teacher_tok, teacher_score, weight),
                          float(temperature), bool(tail))


def distill_step(logits: torch.Tensor, teacher_tok: torch.Tensor, teacher_score: torch.Tensor,
                 temperature: float = 1.0, tail: bool = False,
                 weight: Optional[torch.Tensor] = None, in_place: bool = False):
    """(loss [...], gradient [..., V+1] of its sum) in one pass over the logits;
    ``in_place`` writes the gradient over the logits (a backward pass that needs
    them afterwards raises an error)."""
    tok, score, weight = _teacher(logits, teacher_tok, teacher_score, weight)
    z = logits.detach() if in_place else _even(logits.detach())
    loss = torch.empty(z.shape[:-1], dtype=torch.float32, device=z.device)
    grad = z if in_place else torch.empty(z.shape, dtype=z.dtype, device=z.device)
    capi.tb_distill(z, tok, score, loss, grad, weight=weight, temperature=float(temperature),
                    tail=bool(tail))
    if in_place and not z.is_inference():
        # the library writes by address: a backward pass that still needs these
        # logits finds out by their version
        torch.autograd.graph.increment_version(z)
    return loss, grad

"""The differentiable layer over the row operators where a gradient could be
wrong without a word: second derivatives, logits overwritten before their
backward pass, teachers and weights that ask for a gradient, lists of more
places than a call takes."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def inputs(n=6, C=301, K=5, dtype=F32, seed=0):
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn((n, C), generator=g) * 2).to(dtype).cuda()
    ids = torch.stack([torch.randperm(C, generator=g)[:K] for _ in range(n)]).to(torch.int32)
    return z, ids.cuda(), torch.randn((n, K), generator=g).cuda()


@pytest.mark.parametrize("entry", ["token_scores", "distill_loss"])
def test_second_derivatives_are_refused(entry):
    from paper_2608_21343_amd import rowops
    z, ids, sc = inputs()
    x = z.clone().requires_grad_()
    if entry == "token_scores":
        loss = rowops.token_scores(x, ids).logprob.sum()
    else:
        loss = rowops.distill_loss(x, ids, sc).sum()
    grad, = torch.autograd.grad(loss, x, create_graph=True)
    assert grad.requires_grad  # a penalty on it is not lost on the way ...
    with pytest.raises(RuntimeError, match="second derivative"):
        grad.pow(2).sum().backward()  # ... but refused


@pytest.mark.parametrize("entry", ["token_scores", "distill_loss"])
def test_overwritten_logits_are_noticed(entry):
    from paper_2608_21343_amd import rowops
    z, ids, sc = inputs()
    x = z.clone().requires_grad_()
    y = x * 1.0
    if entry == "token_scores":
        loss = rowops.token_scores(y, ids).logprob.sum()
    else:
        loss = rowops.distill_loss(y, ids, sc).sum()
    rowops.distill_step(y, ids, sc, in_place=True)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_steps_in_place():
    """Without a graph that needs the logits a step in place is an ordinary one."""
    from paper_2608_21343_amd import rowops
    z, ids, sc = inputs()
    loss, grad = rowops.distill_step(z, ids, sc)
    for mode in (torch.enable_grad, torch.no_grad, torch.inference_mode):
        with mode():
            over = z.clone()
            loss2, grad2 = rowops.distill_step(over, ids, sc, in_place=True)
            assert grad2.data_ptr() == over.data_ptr()
            assert bool((loss2 == loss).all()) and bool((over == grad).all())
    over = z.clone()
    with torch.inference_mode():
        rowops.distill_step(over, ids, sc, in_place=True)
    assert bool((over == grad).all())


def test_teachers_and_weights_that_ask_for_a_gradient():
    from paper_2608_21343_amd import rowops
    z, ids, sc = inputs()
    x = z.clone().requires_grad_()
    w = torch.ones(6, device="cuda")
    for kw, word in (({"teacher_score": sc.clone().requires_grad_()}, "teacher_score"),
                     ({"weight": w.clone().requires_grad_()}, "weight")):
        args = {"teacher_score": sc, "weight": w, **kw}
        with pytest.raises(ValueError, match=word):
            rowops.distill_loss(x, ids, **args)
        with pytest.raises(ValueError, match=word):
            rowops.distill_loss(z, ids, **args)
        with torch.no_grad():
            want = rowops.distill_loss(z, ids, **args)
        got = rowops.distill_loss(x, ids, **{k: v.detach() for k, v in args.items()})
        assert bool((got == want).all())
        got.sum().backward()
    # the gradient that distill_step returns is that of the logits alone
    rowops.distill_step(z, ids, sc.clone().requires_grad_(), weight=w.clone().requires_grad_())


@pytest.mark.parametrize("weighted", [False, True])
def test_incoming_gradients_of_any_layout(weighted):
    """Losses and scores that are used transposed, expanded or in part."""
    from paper_2608_21343_amd import rowops
    z, ids, sc = inputs(12)
    x = z.view(4, 3, -1).clone().requires_grad_()
    tok, score = ids.view(4, 3, 5), sc.view(4, 3, 5)
    w = torch.rand(4, 3, device="cuda") if weighted else None
    f = torch.rand(3, 4, device="cuda")
    for use in (lambda y: (y.transpose(0, 1) * f.reshape(3, 4, *[1] * (y.dim() - 2))).sum(),
                lambda y: y.sum(), lambda y: y[:, 1].sum(), lambda y: y[::2].transpose(0, 1).max()):
        for get in (lambda v: rowops.distill_loss(v, tok, score, weight=w),
                    lambda v: rowops.token_scores(v, tok).logprob,
                    lambda v: rowops.token_scores(v, tok, 3).alt_logprob,
                    lambda v: rowops.token_scores(v, tok[..., 0]).logprob,
                    lambda v: rowops.token_scores(v).lse, lambda v: rowops.token_scores(v).entropy):
            y = get(x)
            got, d = torch.autograd.grad(use(y), [x, y])
            want, = torch.autograd.grad(get(x), x, d.contiguous())
            assert bool((got == want).all())


def close(got, want, size, dtype):
    got, want = got.float().cpu().double().numpy(), want.numpy()
    tol = 1e-5 * size.numpy() + 1e-37 + (2.0 ** -7.99 if dtype == BF16 else 3e-7) * np.abs(want)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])


@pytest.mark.parametrize("J, M", [(24, 40), (25, 40), (40, 40), (64, 64), (64, 1), (1, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_more_places_than_a_list_holds(dtype, J, M):
    """Given tokens and alternatives of up to 64 and of more places together: one
    rounding of the gradient in both, also where the two lists' gradients of a
    token or of the whole row nearly cancel. The tolerance is 1e-5 of the
    magnitudes in 32 bits, and the one rounding to bfloat16."""
    from paper_2608_21343_amd.rowops import token_scores
    z, _, _ = inputs(4, 301, 1, dtype, J)
    g = torch.Generator().manual_seed(M)
    alt = torch.topk(z.float(), M, dim=1, sorted=True).indices.cpu()
    tok = torch.randint(0, 301, (4, J), generator=g)
    same = min(J, M)
    tok[:, :same] = alt[:, :same]
    d_tok = torch.randn((4, J), generator=g)
    d_alt = torch.randn((4, M), generator=g)
    d_alt[:2, :same] = -d_tok[:2, :same] + 0.001  # nearly cancel
    d_ent, d_lse = torch.randn(4, generator=g), torch.randn(4, generator=g)
    x = z.clone().requires_grad_()
    got = token_scores(x, tok.to(torch.int32).cuda(), M, 1.3)
    at = got.alt.cpu().long()
    d_tok[2, 0] = d_alt[2, 0] = 0.0
    ((got.logprob * d_tok.cuda()).sum() + (got.alt_logprob * d_alt.cuda()).sum()
     + (got.entropy * d_ent.cuda()).sum() + (got.lse * d_lse.cuda()).sum()).backward()
    y = z.double().cpu().requires_grad_()
    logp = torch.log_softmax(y / 1.3, 1)
    p = logp.exp()
    ent = -(p * logp).sum(1)
    ((torch.gather(logp, 1, tok) * d_tok.double()).sum()
     + (torch.gather(logp, 1, at) * d_alt.double()).sum() + (ent * d_ent.double()).sum()
     + (torch.logsumexp(y / 1.3, 1) * d_lse.double()).sum()).backward()
    p, logp, ent = p.detach(), logp.detach(), ent.detach()
    size = p * ((d_tok.abs().sum(1) + d_alt.abs().sum(1) + d_lse.abs())[:, None]
                + d_ent.abs()[:, None] * (logp.abs() + ent[:, None]))
    size = size.scatter_add(1, tok, d_tok.abs().double()).scatter_add(1, at, d_alt.abs().double())
    close(x.grad, y.grad, size / 1.3, dtype)

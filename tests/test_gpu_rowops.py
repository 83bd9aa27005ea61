"""The differentiable layer over the row operators, against torch's float64
autograd of the plain formulas, and the example that trains with it.

Tolerances: values as in tests/test_gpu_rows.py (1e-5); a gradient is a sum of
at most 70 terms of the same accuracy and size at most 3."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def plain_scores(z, tok, tau, n_alt):
    logp = torch.log_softmax(z / tau, -1)
    lp = torch.where(tok >= 0, torch.gather(logp, -1, tok.clamp(min=0).long()), 0.0)
    alt = torch.topk(z, n_alt, -1).indices
    return (lp, torch.logsumexp(z / tau, -1), -(logp.exp() * logp).sum(-1),
            torch.gather(logp, -1, alt))


@pytest.mark.parametrize("J, M", [(2, 5), (0, 4), (3, 0), (40, 40)])
def test_token_scores_and_gradient(J, M):
    from paper_2608_21343_amd.rowops import token_scores
    g = torch.Generator().manual_seed(J)
    z = torch.randn((3, 4, 301), generator=g) * 2
    tok = torch.randint(-1, 301, (3, 4, J), generator=g, dtype=torch.int32)
    w = [torch.randn(s, generator=g) for s in ((3, 4, J), (3, 4), (3, 4), (3, 4, M))]
    x = z.cuda().requires_grad_()
    got = token_scores(x, tok.cuda() if J else None, M, 1.4)
    outs = (got.logprob, got.lse, got.entropy, got.alt_logprob)
    sum((o * v.cuda()).sum() for o, v in zip(outs, w)).backward()
    y = z.double().requires_grad_()
    want = plain_scores(y, tok, 1.4, M)
    sum((o * v.double()).sum() for o, v in zip(want, w)).backward()
    for o, v in zip(outs, want):
        np.testing.assert_allclose(o.detach().cpu().numpy(), v.detach().numpy(), atol=1e-5)
    np.testing.assert_allclose(x.grad.cpu().numpy(), y.grad.numpy(), atol=2e-4)


def test_one_token_a_row_and_rows_unevenly_spaced():
    from paper_2608_21343_amd.rowops import token_scores
    z = torch.randn(5, 6, 50).cuda()[:, :4]  # a view whose rows are not evenly spaced
    tok = torch.randint(0, 50, (5, 4), dtype=torch.int32).cuda()
    x = z.detach().requires_grad_()
    got = token_scores(x, tok)
    assert got.logprob.shape == (5, 4) and got.alt.shape == (5, 4, 0)
    got.logprob.sum().backward()
    want = torch.log_softmax(z, -1).gather(-1, tok.long()[..., None])[..., 0]
    torch.testing.assert_close(got.logprob.detach(), want, atol=1e-5, rtol=0)
    hot = torch.nn.functional.one_hot(tok.long(), 50) - torch.softmax(z, -1)
    torch.testing.assert_close(x.grad, hot, atol=1e-5, rtol=0)
    with pytest.raises(ValueError, match="tokens"):
        token_scores(z, tok[:4])


@pytest.mark.parametrize("tail", [False, True])
def test_distill_loss_and_gradient(tail):
    from paper_2608_21343_amd.rowops import distill_loss, distill_step
    g = torch.Generator().manual_seed(5)
    z = torch.randn((4, 3, 200), generator=g)
    ids = torch.stack([torch.randperm(200, generator=g)[:6] for _ in range(12)]).view(4, 3, 6)
    sc = torch.randn((4, 3, 6), generator=g)
    if tail:
        sc = torch.log_softmax(sc, -1) - 0.3
    w, d = torch.rand((4, 3), generator=g), torch.randn((4, 3), generator=g)
    x = z.cuda().requires_grad_()
    args = (ids.to(torch.int32).cuda(), sc.cuda())
    loss = distill_loss(x, *args, temperature=1.2, tail=tail, weight=w.cuda())
    (loss * d.cuda()).sum().backward()
    y = z.double().requires_grad_()
    logp = torch.log_softmax(y / 1.2, -1)
    logq = sc.double() if tail else torch.log_softmax(sc.double() / 1.2, -1)
    lp = torch.gather(logp, -1, ids)
    want = (logq.exp() * (logq - lp)).sum(-1)
    if tail:
        rest = 1 - logq.exp().sum(-1)
        want = want + rest * (rest.log() - (1 - lp.exp().sum(-1)).log())
    want = want * w
    (want * d).sum().backward()
    np.testing.assert_allclose(loss.detach().cpu().numpy(), want.detach().numpy(), atol=1e-5)
    np.testing.assert_allclose(x.grad.cpu().numpy(), y.grad.numpy(), atol=1e-5)
    both, grad = distill_step(x, *args, temperature=1.2, tail=tail, weight=w.cuda())
    torch.testing.assert_close(both, loss.detach(), atol=0, rtol=0)
    over = z.cuda()
    _, same = distill_step(over, *args, temperature=1.2, tail=tail, weight=w.cuda(), in_place=True)
    assert same.data_ptr() == over.data_ptr()
    torch.testing.assert_close(same, grad, atol=0, rtol=0)


def test_example_learns():
    import importlib.util
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location(
        "train_from_teacher", os.path.join(root, "examples", "train_from_teacher.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last = example.main(steps=12, B=8, T=16, quiet=True)
    assert np.isfinite(first) and last < 0.7 * first

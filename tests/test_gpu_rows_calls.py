"""Row operators: calls without rows, workspaces on other streams, and rows
whose results do not depend on their place or number."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_calls_without_rows():
    from paper_2608_21343_amd import capi
    from paper_2608_21343_amd.rowops import distill_loss, token_scores
    z = torch.empty((0, 301), device="cuda", requires_grad=True)
    tok = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    got = token_scores(z, tok, 4)
    assert got.logprob.shape == (0, 2) and got.alt.shape == (0, 4) and got.lse.shape == (0,)
    loss = distill_loss(z, tok, torch.empty((0, 2), device="cuda"))
    (got.logprob.sum() + loss.sum()).backward()
    assert z.grad.shape == (0, 301)
    assert capi.tb_rows_workspace_bytes(z.detach(), 8) == 0


@pytest.mark.parametrize("C", [140001, 400003])
def test_workspace_of_another_stream(C):
    """A call on a given stream whose workspace the binding allocates: work queued
    on the current stream right after it does not take that memory."""
    from paper_2608_21343_amd import capi
    g = torch.Generator(device="cuda").manual_seed(C)
    z = torch.randn((40, C), generator=g, device="cuda")
    alt = torch.empty((40, 16), dtype=torch.int32, device="cuda")
    alt_lp = torch.empty((40, 16), device="cuda")
    want = torch.topk(z, 16, dim=1).indices
    side = torch.cuda.Stream()
    for _ in range(3):
        alt.fill_(-5)
        torch.cuda.synchronize()
        capi.tb_token_logprobs(z, out_alt=alt, out_alt_logprob=alt_lp, stream=side)
        need = capi.tb_rows_workspace_bytes(z, 16)
        assert need > 0
        junk = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert bool((alt == want).all())
        del junk


@pytest.mark.parametrize("dtype, C", [(torch.float32, 1025), (torch.float32, 4097),
                                      (torch.bfloat16, 1025), (torch.bfloat16, 8193)])
def test_rows_of_one_wave_do_not_depend_on_place_or_number(dtype, C):
    from paper_2608_21343_amd import capi
    g = torch.Generator().manual_seed(C)
    few = (torch.randn((7, C), generator=g) * 2).to(dtype).cuda()
    many = few.repeat(700, 1)
    many = torch.nn.functional.pad(many, (0, 3))[:, :C]  # other places in memory
    tok = torch.randint(0, C, (7, 2), generator=g, dtype=torch.int32).cuda()
    out = []
    for z, t in ((few, tok), (many, tok.repeat(700, 1))):
        n = z.shape[0]
        lp, lse, ent = (torch.empty(s, device="cuda") for s in ((n, 2), (n,), (n,)))
        alt = torch.empty((n, 8), dtype=torch.int32, device="cuda")
        alt_lp = torch.empty((n, 8), device="cuda")
        capi.tb_token_logprobs(z, t, lp, lse, ent, alt, alt_lp)
        loss, grad = torch.empty(n, device="cuda"), torch.empty((n, C), dtype=dtype, device="cuda")
        capi.tb_distill(z, alt, alt_lp, loss, grad, temperature=1.5)
        out.append([x.cpu() for x in (lp, lse, ent, alt, alt_lp, loss, grad)])
    for a, b in zip(*out):
        bits = (lambda x: x.view(torch.int32 if x.dtype != torch.bfloat16 else torch.int16))
        np.testing.assert_array_equal(bits(a).repeat(*([700] + [1] * (a.dim() - 1))).numpy(),
                                      bits(b).numpy())


@pytest.mark.parametrize("z_out", [-86.0, -87.2, -87.33, -100.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tail_of_almost_no_mass(dtype, z_out):
    """One token outside the list has the least probability that float32 holds
    (or less), all others none: its gradient takes the teacher's whole rest, and
    the tokens of probability 0 have none. Its exponential is within 3 roundings
    of its exponent, 87 * 2^-22, of the true one, but the quotient by their sum,
    which is itself, is exact; below 2^-126 it counts as 0 and the loss as inf."""
    from paper_2608_21343_amd import capi
    C = 300
    z = torch.full((2, C), -float("inf"))
    z[:, :40] = 0.0
    z[:, 250] = z_out
    z = z.to(dtype).cuda()
    ids = torch.arange(40, dtype=torch.int32).repeat(2, 1).cuda()
    sc = torch.full((2, 40), float(np.log(0.5 / 40))).cuda()
    loss, grad = torch.empty(2, device="cuda"), torch.empty_like(z)
    capi.tb_distill(z, ids, sc, loss, grad, tail=True)
    g = grad.float().cpu().numpy()
    low = float(z[0, 250]) < -87.336  # 126 ln 2
    tol = 2.0 ** -8 if dtype == torch.bfloat16 else 1e-5
    np.testing.assert_allclose(g[:, :40], 1 / 40 - 0.5 / 40, atol=1e-6 + tol / 80)
    rest = np.delete(g[:, 40:], 210, 1)
    assert (rest == 0).all()
    if low:
        assert np.isinf(loss.cpu().numpy()).all() and (np.abs(g[:, 250]) < 1e-30).all()
    else:
        np.testing.assert_allclose(g[:, 250], -0.5, atol=0.5 * tol + 1e-5)
        want = 0.5 * (np.log(0.5 / 40) - np.log(1 / 40)) + 0.5 * (
            np.log(0.5) - (float(z[0, 250]) - np.log(40)))
        np.testing.assert_allclose(loss.cpu().numpy(), want, atol=5e-5)

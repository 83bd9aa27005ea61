"""The output layer under autograd where a training program meets it: batches without
rows, rows that are nearly certain, captures."""

import pytest
import torch

from tests import linear_reference as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(0,), (0, 5), (3, 0)])
def test_a_batch_without_rows(shape, dtype):
    """Losses of that shape, and gradients of 0."""
    from paper_2608_21343_amd import capi
    from paper_2608_21343_amd.linearops import linear_xent, linear_xent_step
    c = R.case(4, 64, 300, dtype, 1, device="cuda")
    x = torch.zeros((*shape, 64), dtype=dtype, device="cuda", requires_grad=True)
    w, b = (c[k].clone().requires_grad_() for k in ("w", "bias"))
    target = torch.zeros(shape, dtype=torch.int32, device="cuda")
    out = linear_xent(x, w, target, b, torch.ones(shape, device="cuda"))
    assert out.loss.shape == out.lse.shape == shape
    (out.loss.sum() + out.lse.sum()).backward()
    assert x.grad.shape == x.shape and w.grad.shape == w.shape
    assert not w.grad.any() and not b.grad.any()
    x.grad = None
    linear_xent(x, c["w"], target).loss.sum().backward()  # features alone
    assert x.grad.shape == x.shape
    loss, dx, dw, db = linear_xent_step(x.detach(), c["w"], target, c["bias"])
    assert loss.shape == shape and dx.shape == x.shape and not dw.any() and not db.any()
    capi.tb_linear_xent(x.detach(), c["w"], target, loss)


@pytest.mark.parametrize("dtype, n", [(F32, 9), (F32, 16), (F32, 17), (F32, 32), (F32, 33),
                                      (F32, 64), (F32, 65), (BF16, 9), (BF16, 16), (BF16, 17),
                                      (BF16, 32), (BF16, 33)])
def test_both_passes_see_the_same_logits(dtype, n):
    """Rows that are nearly certain, of values whose logits depend on how they are summed:
    lse has to be that of the logits which the backward pass makes, or p - 1 is their
    difference.

    float32: 1 + 2^-12 + 2^-23 takes 24 bits; two float16 planes hold 23 of them, so 1024
    of them are short by 2^-13, of all tokens alike. Among each other the logits may be off by
    e = 2^-5 + 2^-13: the target's sum is of multiples of 2^-12 below 2^11, exact in any order;
    the others' is of 1024 products 2^-12 (1 - 2^-6) of the lower plane besides, and if each is
    added on its own, each addition rounds by half a step of a sum below 1024, 2^-15.
    bfloat16: 32 sums of 32 products, each 3/8 of a step of a sum of 1024, which a sum that
    begins at the bias drops and one to which the bias is added keeps, for all tokens alike;
    e = 2^-12, a rounding or two of half a step of 1024, 2^-14 each."""
    from paper_2608_21343_amd.linearops import linear_xent
    D, C, at = 1024, 1025, 5
    if dtype == F32:
        x = torch.full((n, D), 1 + 2.0 ** -12 + 2.0 ** -23, device="cuda")
        w = torch.full((C, D), 1 - 2.0 ** -6, device="cuda")
        w[at] = 1.0
        b = torch.zeros(C, device="cuda")
    else:
        x = torch.full((n, D), 3 * 2.0 ** -11, dtype=dtype, device="cuda")
        w = torch.full((C, D), 2.0 ** -10, dtype=dtype, device="cuda")
        b = torch.full((C,), 1024.0, dtype=dtype, device="cuda")
        b[at] = 1040.0
    target = torch.full((n,), at, dtype=torch.int32, device="cuda")
    z = x[:1].double() @ w.double().t() + b.double()
    p = torch.softmax(z, 1)[0]
    G = p * n
    rest = 1 - p[at]
    G[at] = -(p.sum() - p[at]) * n
    assert 1e-5 < float(rest) < 1e-3
    leaves = [t.requires_grad_() for t in (x, w, b)]
    _, dw, db = torch.autograd.grad(linear_xent(*leaves[:2], target, b).loss.sum(), leaves)
    # the logits' differences (e^2e - 1, below 4 e), exponentials of -16 to 2^-19 of themselves,
    # n additions; for the target's entry roundings near 1 besides: four of a, and of the sum of
    # the 64 tokens beside it
    e = 2.0 ** -12 if dtype == BF16 else 2.0 ** -5 + 2.0 ** -13
    tol = G.abs() * (4 * e + 2.0 ** -18 + (n + 4) * 2.0 ** -24)
    tol[at] += n * (4 + 68) * 2.0 ** -24
    off = (db.double() - G).abs()
    assert bool((off <= tol + R.U[dtype] * G.abs()).all()), (off / G.abs()).max()
    # (x is one value; G's own rounding is a part of b with many bfloat16 rows, of G with others)
    one = float(x[0, 0].detach())
    planes = R.U[dtype] if dtype == BF16 else 2.0 ** -21
    off = (dw.double() - G[:, None] * one).abs()
    assert bool((off <= one * (tol + (planes + R.U[dtype]) * G.abs())[:, None]).all()), off.max()


def layer(n=100, dtype=BF16):
    """Features and float32 weights that are cast for the call, and a pass through it."""
    from paper_2608_21343_amd.linearops import linear_xent
    c = R.case(n, 64, 500, dtype, 16, device="cuda")
    x = c["x"].float().requires_grad_()
    w = c["w"].float().requires_grad_()

    def run():
        loss = linear_xent(x.to(dtype), w.to(dtype), c["target"], c["bias"]).loss.sum()
        return (loss, *torch.autograd.grad(loss, (x, w)))

    return run


def test_a_capture_beside_an_eager_loss_is_refused():
    """The leaves lie behind casts; the loss is of the default stream."""
    run = layer()
    loss = run()[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="drop its losses"):
            run()
    del loss


def test_a_capture_beside_its_warm_up():
    """The usual recipe: some passes on a side stream, whose last loss is still in scope."""
    run = layer()
    want = [t.detach().clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            loss, dx, dw = run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        for t in out[1:]:
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((a == b).all()) for a, b in zip(out[1:], want[1:]))
        run()
    assert torch.isfinite(loss)

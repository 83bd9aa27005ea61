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

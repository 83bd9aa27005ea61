"""The float64 form of the output layer's cross entropy against autograd and
differences, and the refusals of its calls (no GPU is needed for either)."""

import numpy as np
import pytest
import torch

from tests import linear_reference as R


def doubles(c):
    return {k: v if v is None or v.dtype == torch.int32 else v.double() for k, v in c.items()}


@pytest.mark.parametrize("weighted, gaps, bias", [(False, False, True), (True, True, False)])
def test_reference_against_autograd(weighted, gaps, bias):
    c = doubles(R.case(9, 5, 12, torch.float32, 1, bias, weighted, gaps))
    g = torch.Generator().manual_seed(2)
    d_loss, d_lse = torch.randn((2, 9), generator=g, dtype=torch.float64)
    leaves = [t.requires_grad_() for t in (c["x"], c["w"], c["bias"]) if t is not None]
    loss, lse, z = R.forward(**c)
    got = torch.autograd.grad((loss * d_loss + lse * d_lse).sum(), leaves)
    G = R.logit_grad(z.detach(), lse.detach(), c["target"], c["weight"], d_loss, d_lse)
    # a row that is left out has lse 0 whatever its logits are
    x, w = c["x"].detach(), c["w"].detach()
    assert torch.allclose(got[0], G @ w, atol=1e-12)
    assert torch.allclose(got[1], G.t() @ x, atol=1e-12)
    if bias:
        assert torch.allclose(got[2], G.sum(0), atol=1e-12)


def test_reference_against_differences():
    c = doubles(R.case(6, 4, 7, torch.float32, 3, True, True, False))
    loss, lse, z = R.forward(**c)
    G = R.logit_grad(z, lse, c["target"], c["weight"])
    for name, grad in (("x", G @ c["w"]), ("w", G.t() @ c["x"]), ("bias", G.sum(0))):
        flat = c[name].view(-1) if c[name].is_contiguous() else None
        assert flat is not None
        for i in range(0, flat.numel(), 3):
            at, h = flat[i].item(), 1e-5
            flat[i] = at + h
            up = R.forward(**c)[0].sum()
            flat[i] = at - h
            down = R.forward(**c)[0].sum()
            flat[i] = at
            assert abs((up - down) / (2 * h) - grad.reshape(-1)[i]) < 1e-8


# ---- refusals: the arguments are checked before any launch

P = 1 << 20  # an aligned address that nothing reads
BIG = 1 << 40


def xent(lib, **change):
    a = dict(x=P, w=2 * P, bias=0, dtype=1, n=4, D=64, V1=100, xs=64, ws=64, target=3 * P,
             weight=0, loss=4 * P, lse=5 * P, low=0, dx=0, dxs=64, dw=0, dws=64, db=0, wk=6 * P,
             wkb=BIG, st=0)
    a.update(change)
    return lib.tb_linear_xent(*a.values())


def xent_grad(lib, **change):
    a = dict(x=P, w=2 * P, bias=0, dtype=1, n=4, D=64, V1=100, xs=64, ws=64, target=3 * P,
             weight=0, lse=4 * P, low=0, dl=0, dls=1, dlse=0, dx=7 * P, dxs=64, dw=0,
             dws=64, db=0, wk=9 * P, wkb=BIG, st=0)
    a.update(change)
    return lib.tb_linear_xent_grad(*a.values())


REFUSED = [
    (dict(dtype=2), "dtype"), (dict(n=-1), "n_rows"), (dict(n=(1 << 24) + 1), "n_rows"),
    (dict(D=0), "width"), (dict(D=(1 << 16) + 1), "width"), (dict(V1=1), "v_plus_blank"),
    (dict(V1=(1 << 20) + 1), "v_plus_blank"), (dict(ws=63), "w_stride"),
    (dict(xs=63), "x_stride"), (dict(x=0), "x is NULL"), (dict(w=0), "w is NULL"),
    (dict(x=P + 1), "x misaligned"), (dict(w=P + 1), "w misaligned"),
    (dict(bias=P + 1), "bias misaligned"), (dict(target=0), "target is NULL"),
    (dict(target=P + 2), "target"), (dict(weight=P + 2), "weight"),
    (dict(dx=8 * P, dxs=63), "dx_stride"), (dict(dw=8 * P + 1), "dw misaligned"),
    (dict(dw=8 * P, dws=63), "dw_stride"), (dict(db=8 * P + 1), "db misaligned"),
    (dict(wk=0), "workspace holds 0"), (dict(wkb=1000), "workspace holds 1000"),
    (dict(wk=9 * P + 16), "workspace not 256"), (dict(dx=P), "dx overlaps x"),
    (dict(dw=2 * P), "dw overlaps w"), (dict(db=3 * P), "db overlaps target"),
    (dict(dx=8 * P, dw=8 * P), "dx overlaps dw"),
]


@pytest.mark.parametrize("change, message", REFUSED)
def test_refusals(change, message):
    from paper_2608_21343_amd import capi
    for call in (xent, xent_grad):
        assert call(capi.LIB, **change) != 0
        assert message in capi.LIB.tb_last_error().decode()


def test_refusals_of_either():
    from paper_2608_21343_amd import capi
    for call, change, message in (
            (xent, dict(loss=0, lse=0), "every output"), (xent, dict(loss=4 * P + 2), "out_loss"),
            (xent, dict(lse=4 * P), "out_loss overlaps out_lse"),
            (xent, dict(wk=4 * P), "overlaps workspace"),
            (xent, dict(low=5 * P + 2), "out_low"),
            (xent, dict(low=5 * P), "out_lse overlaps out_low"),
            (xent_grad, dict(low=P + 2), "lse_low"),
            (xent_grad, dict(low=7 * P), "dx overlaps lse_low"),
            (xent_grad, dict(dx=0), "all NULL"), (xent_grad, dict(lse=0), "lse is NULL"),
            (xent_grad, dict(dls=2), "d_loss_step"),
            (xent_grad, dict(dl=7 * P, dls=0), "dx overlaps d_loss"),
            (xent_grad, dict(dl=P + 2), "d_loss"), (xent_grad, dict(dlse=P + 2), "d_lse"),
            (xent_grad, dict(dx=4 * P), "dx overlaps lse")):
        assert call(capi.LIB, **change) != 0
        assert message in capi.LIB.tb_last_error().decode()


def test_calls_without_rows_touch_nothing():
    from paper_2608_21343_amd import capi
    assert xent(capi.LIB, n=0, x=0, w=0, target=0, loss=8, lse=8, wk=0, wkb=0) == 0


def test_workspace_bytes():
    from paper_2608_21343_amd import capi
    f = capi.LIB.tb_linear_xent_workspace_bytes
    used = f(1, 1000, 640, 8193, P, 640, 0, 0)
    # float32 operands and odd widths need a copy of the weights
    assert f(1, 1000, 640, 8193, P + 2, 640, 0, 0) >= used + 8193 * 640 * 2
    assert f(1, 1000, 639, 8193, P, 640, 0, 0) >= used + 8193 * 640 * 2
    # the gradients of the logits take pieces, not all of them
    whole = f(1, 1 << 16, 256, 1 << 20, P, 256, 3, 1)
    assert 0 < whole < (1 << 16) * (1 << 20) * 2 // 8
    # without rows dw and db are still written
    assert 0 < f(1, 0, 640, 8193, P, 640, 7, 0) and 0 < f(0, 0, 1, 2, 0, 1, 7, 1)
    for bad in ((2, 1, 1, 2, P, 1, 0, 0), (1, -1, 1, 2, P, 1, 0, 0), (1, 1, 1, 2, P, 1, 8, 0),
                (1, 1, 1, 2, P, 1, 0, 2), (1, 1, 1, 1, P, 1, 0, 0)):
        assert f(*bad) == -1


def adamw(lib, change=None, tensor=None, count=2):
    rec = np.zeros((count, 8), dtype=np.int64)
    for k in range(count):
        rec[k] = [(8 * k + i + 1) * P for i in range(7)] + [1000]
        rec[k, 4:7] = 0
    for (k, i), value in (tensor or {}).items():
        rec[k, i] = value
    a = dict(t=rec.ctypes.data, n=count, dtype=0, bits=32, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8,
             wd=0.01, step=1, lrd=0, sd=0, gs=0, seed=0, st=0)
    a.update(change or {})
    return lib.tb_adamw_step(*a.values())


@pytest.mark.parametrize("change, tensor, message", [
    (dict(n=-1), {}, "tensors"), (dict(t=0), {}, "tensors"), (dict(dtype=2), {}, "dtype"),
    (dict(bits=16), {}, "state_bits"), (dict(lr=-1.0), {}, "lr"),
    (dict(lr=float("nan")), {}, "lr"), (dict(lr=float("inf")), {}, "lr"),
    (dict(wd=-1.0), {}, "weight_decay"), (dict(eps=-1.0), {}, "eps"),
    (dict(b1=1.0), {}, "beta1"), (dict(b2=-0.1), {}, "beta2"), (dict(step=0), {}, "step"),
    (dict(lrd=P + 2), {}, "lr_dev"), (dict(sd=P + 4), {}, "step_dev"),
    (dict(gs=P + 1), {}, "grad_scale"),
    ({}, {(1, 7): -1}, "tensor 1"), ({}, {(1, 7): (1 << 36) + 1}, "tensor 1"),
    ({}, {(0, 0): 0}, "param"), ({}, {(1, 0): P + 2}, "param"), ({}, {(0, 1): 0}, "grad"),
    ({}, {(0, 2): 0}, "m is NULL"), ({}, {(0, 3): P + 1}, "v is NULL or not"),
    (dict(bits=8), {}, "m_unit"), (dict(bits=8), {(0, 4): 20 * P}, "v_unit"),
    ({}, {(0, 6): 20 * P}, "master"), (dict(dtype=1), {(0, 6): 20 * P}, "some tensors only"),
    # the same parameter twice, a gradient in another's state, one value of overlap
    ({}, {(1, 0): P}, "shares memory"), ({}, {(1, 1): 3 * P}, "shares memory"),
    ({}, {(1, 2): P + 4 * 999}, "shares memory"), (dict(lrd=P), {}, "shares memory"),
])
def test_adamw_refusals(change, tensor, message):
    from paper_2608_21343_amd import capi
    assert adamw(capi.LIB, change, tensor) != 0
    assert message in capi.LIB.tb_last_error().decode()


def test_adamw_calls_without_values():
    from paper_2608_21343_amd import capi
    assert adamw(capi.LIB, {"n": 0, "t": 0}) == 0
    none = {(k, i): 0 for k in range(2) for i in range(8)}
    assert adamw(capi.LIB, {}, none) == 0


def test_adamw_moments_refusals():
    from paper_2608_21343_amd import capi
    rec = np.zeros((2, 8), dtype=np.int64)
    for k in range(2):
        rec[k] = [(8 * k + i + 1) * P for i in range(7)] + [1000]
    out_m = np.array([30 * P, 31 * P], dtype=np.int64)
    out_v = np.array([32 * P, 33 * P], dtype=np.int64)

    def call(n=2):
        return capi.LIB.tb_adamw_moments(rec.ctypes.data, n, out_m.ctypes.data,
                                         out_v.ctypes.data, 0)

    for array, at, value, message in ((rec, (0, 2), 0, "m is NULL"), (rec, (1, 3), 0, "v is NULL"),
                                      (rec, (0, 4), P + 2, "m_unit"), (rec, (0, 5), 0, "v_unit"),
                                      (out_m, 1, 0, "out_m"), (out_v, 0, P + 2, "out_v"),
                                      (out_m, 1, 30 * P + 4, "shares memory"),
                                      (out_v, 1, 3 * P, "shares memory"),
                                      (rec, (0, 7), -1, "tensor 0")):
        keep = array[at]
        array[at] = value
        assert call() != 0
        assert message in capi.LIB.tb_last_error().decode()
        array[at] = keep
    assert call(-1) != 0


def test_captures_beside_an_eager_graph_are_refused(monkeypatch):
    """The check alone, without a capture: a leaf whose eager graph is alive."""
    from paper_2608_21343_amd import linearops
    x, w = torch.zeros(3, requires_grad=True), torch.zeros(3)
    capturing = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    y = x * w
    linearops._mark(y.grad_fn)
    capturing[0] = True
    again = x * w
    with pytest.raises(RuntimeError, match="drop its losses"):
        linearops._mark(again.grad_fn)
    del y, again
    y = x * w
    linearops._mark(y.grad_fn)
    linearops._mark((x * w).grad_fn)  # further calls of one capture
    del y


def test_first_steps_are_not_captured(monkeypatch):
    """States made inside a capture would be empty again in every replay."""
    from paper_2608_21343_amd import optim
    p = torch.zeros(3, requires_grad=True)
    p.grad = torch.ones(3)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for capturable in (False, True):
        with pytest.raises(RuntimeError, match="before the capture"):
            optim.AdamW([p], capturable=capturable).step()


def test_workspace_of_far_rows():
    """Weights whose rows lie more than 2^22 values apart are copied."""
    from paper_2608_21343_amd import capi
    f = capi.LIB.tb_linear_xent_workspace_bytes
    for grads in (0, 7):
        near, far = (f(1, 1000, 640, 8193, P, stride, grads, 0)
                     for stride in (1 << 22, (1 << 22) + 8))
        assert 8193 * 640 * 2 <= far - near <= 8193 * 640 * 2 + 256

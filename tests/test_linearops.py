"""Which captures the output layer refuses, without a GPU: the check alone, on graphs
of the host."""

import gc

import pytest
import torch

from paper_2608_21343_amd import linearops


@pytest.fixture
def capturing(monkeypatch):
    now = [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now[0])
    gc.collect()
    return now


def model(w, u):
    """Weights that reach the call through a cast and a transpose, features through layers."""
    x = torch.ones(4, 3)
    for _ in range(3):
        x = torch.tanh(x @ u)
    return (x.bfloat16() @ w.bfloat16().t()).float()


@pytest.mark.parametrize("shared", ["w", "u"])
def test_leaves_behind_other_nodes_are_seen(shared, capturing):
    w, u = torch.ones(5, 3, requires_grad=True), torch.ones(3, 3, requires_grad=True)
    eager = model(w if shared == "w" else w.detach(), u if shared == "u" else u.detach())
    linearops._mark(eager.grad_fn)
    capturing[0] = True
    with pytest.raises(RuntimeError, match="drop its losses"):
        linearops._mark(model(w, u).grad_fn)
    del eager
    captured = model(w, u)
    linearops._mark(captured.grad_fn)
    linearops._mark(model(w, u).grad_fn)


def test_other_leaves_are_no_hindrance(capturing):
    w, u, v = (torch.ones(3, 3, requires_grad=True) for _ in range(3))
    eager = model(w, u)
    linearops._mark(eager.grad_fn)
    capturing[0] = True
    linearops._mark(model(v, v).grad_fn)


def test_a_loss_of_a_loop_is_forgotten_with_its_graph(capturing):
    w, u = torch.ones(5, 3, requires_grad=True), torch.ones(3, 3, requires_grad=True)
    for _ in range(4):
        loss = model(w, u)
        linearops._mark(loss.grad_fn)
        loss.sum().backward()
    assert len(linearops._eager) >= 1
    del loss
    assert not linearops._eager


def test_warm_up_on_a_side_stream(capturing, monkeypatch):
    """A side stream can join a capture, so a loss of a warm-up there may be in scope."""
    w, u = torch.ones(5, 3, requires_grad=True), torch.ones(3, 3, requires_grad=True)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(linearops.capi, "_stream", lambda stream: 1)
    warm = model(w, u)
    linearops._mark(warm.grad_fn)
    capturing[0] = True
    linearops._mark(model(w, u).grad_fn)

"""The torch optimizer's own work, without a GPU: the library's step is replaced by one that
notes its arguments."""

import pytest
import torch

from paper_2608_21343_amd import optim


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(optim.capi, "tb_adamw_step",
                        lambda param, *a, **how: made.append(dict(how, param=param)))
    return made


def leaf(n=3):
    p = torch.zeros(n, requires_grad=True)
    p.grad = torch.ones(n)
    return p


def test_only_capturable_steps_are_captured(calls, monkeypatch):
    """A captured graph would hold the number of the step, and with it the bias
    corrections and roundings, of its capture."""
    one, two = leaf(), leaf()
    opt = optim.AdamW([dict(params=[one], capturable=True), dict(params=[two])])
    opt.step()
    opt.step()
    done, step = len(calls), opt.state[two]["step"]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="capturable"):
        opt.step()
    assert len(calls) == done and opt.state[two]["step"] == step  # nothing has moved
    opt.param_groups[1]["params"][0].grad = None
    with pytest.raises(RuntimeError, match="capturable"):
        opt.step()
    alone = leaf()
    opt = optim.AdamW([alone], capturable=True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    opt.step()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    opt.step()
    assert len(calls) == done + 2

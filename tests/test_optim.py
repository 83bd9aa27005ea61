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


@pytest.fixture
def steps(monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(optim.capi, "tb_adamw_step",
                        lambda param, *a, step, step_dev, **how: made.append(
                            step if step_dev is None else (int(step_dev), step_dev.device)))
    return made


def test_counters_resume_on_their_parameters_device(steps, tmp_path):
    """A state dict of other devices than those of the parameters: the counter goes on."""
    one, two = leaf(), leaf(5)
    opt = optim.AdamW([one, two], lr=torch.tensor(1e-3), capturable=True)
    for _ in range(2):
        opt.step()
    saved = opt.state_dict()
    here = torch.device("cpu")
    group = saved["param_groups"][0]
    assert group["step_dev"][here].tolist() == [2]
    other = dict(saved, param_groups=[dict(group, step_dev={
        torch.device("meta"): group["step_dev"][here].clone()})])
    torch.save(saved, tmp_path / "state.pt")
    for state in (saved, other, torch.load(tmp_path / "state.pt", map_location="cpu",
                                           weights_only=True)):
        again = optim.AdamW([leaf(), leaf(5)], capturable=True)
        again.load_state_dict(state)
        steps.clear()
        again.step()
        assert steps == [(3, here)]
        assert again.param_groups[0]["step_dev"].keys() == {here}
    assert group["step_dev"][here].tolist() == [2]  # the saved one stays


def test_capturable_may_change(steps, monkeypatch):
    """The number of steps goes along, both ways."""
    one, two = leaf(), leaf(5)
    opt = optim.AdamW([one, two])
    for _ in range(3):
        opt.step()
    opt.param_groups[0]["capturable"] = True
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="before the capture"):
        opt.step()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    opt.step()
    opt.step()
    opt.param_groups[0]["capturable"] = False
    opt.step()
    assert steps == [1, 2, 3, (4, one.device), (5, one.device), 6]
    one.grad = None
    opt.step()
    one.grad = torch.ones(3)
    opt.param_groups[0]["capturable"] = True
    with pytest.raises(RuntimeError, match="different numbers"):
        opt.step()


@pytest.mark.parametrize("group, message", [
    (dict(params=[torch.zeros(4, dtype=torch.float16)]), "float32 or bfloat16"),
    (dict(params=[torch.zeros(4, 6).t()]), "contiguous"),
    (dict(params=[torch.zeros(4)], state_bits=4), "state_bits"),
    (dict(params=[torch.zeros(4)], lr=torch.zeros(2)), "learning rate"),
])
def test_a_group_that_is_refused_leaves_nothing(group, message, calls):
    group["params"][0].requires_grad_()
    kept = leaf()
    opt = optim.AdamW([kept])
    with pytest.raises(ValueError, match=message):
        opt.add_param_group(group)
    assert len(opt.param_groups) == 1
    opt.step()
    assert len(calls) == 1 and calls[0]["param"][0] is kept
    with pytest.raises(ValueError, match=message):
        optim.AdamW([group])

"""The torch optimizer on the GPU: a capturable run that goes on from a saved state."""

import pytest
import torch

from tests.test_gpu_adamw import KINDS, layers, set_grads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, bits, master", KINDS)
def test_a_capturable_run_resumes(dtype, bits, master, tmp_path):
    """Through a file that is loaded to the host: bit for bit as without it, captured."""
    from paper_2608_21343_amd.optim import AdamW

    def make(params):
        return AdamW(params, lr=torch.tensor(1e-2, device="cuda"), state_bits=bits, master=master,
                     capturable=True, seed=5)

    one = layers(dtype)
    a = make(one)
    for turn in range(3):
        set_grads(one, turn)
        a.step()
    torch.save(a.state_dict(), tmp_path / "state.pt")
    two = [torch.nn.Parameter(p.detach().clone()) for p in one]
    b = make(two)
    b.load_state_dict(torch.load(tmp_path / "state.pt", map_location="cpu", weights_only=True))
    for turn in range(3, 5):
        for params, opt in ((one, a), (two, b)):
            set_grads(params, turn)
            opt.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for turn in range(5, 9):
        set_grads(one, turn)
        a.step()
        for p, q in zip(one, two):
            q.grad.copy_(p.grad)
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(one, two):
            assert bool((p == q).all()), turn
            for name, t in a.state[p].items():
                if isinstance(t, torch.Tensor):
                    assert bool((b.state[q][name] == t).all()), name

"""The output layer's calls write nothing behind the workspace that they ask for."""

import pytest
import torch

from tests import linear_reference as R
from tests.test_gpu_linear import check_all, outputs

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
BEHIND = 1 << 20  # bytes that are watched


def guarded(need, fill):
    """A workspace of `need` bytes, and all of its buffer: what surrounds it is 0xa5."""
    whole = torch.full((256 + need + BEHIND,), 0xa5, dtype=torch.uint8, device="cuda")
    whole[256:256 + need] = fill
    return whole[256:256 + need], whole


def untouched(whole, need):
    return bool((whole[:256] == 0xa5).all()) and bool((whole[256 + need:] == 0xa5).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D, C", [(64, 300), (65, 64), (512, 1025), (1024, 257)])
@pytest.mark.parametrize("n", [0, 1, 2, 16, 17, 32, 33, 64, 65, 257, 3000])
def test_nothing_is_written_behind_the_workspace(n, D, C, dtype):
    from paper_2608_21343_amd import capi
    c = R.case(n, D, C, dtype, 2, device="cuda", weighted=True, gaps=True)
    want = R.expected(c) if n else None
    lse = torch.zeros(n, device="cuda")
    for names in (("dw",), ("db",), ("dw", "db"), ("dx", "dw", "db"), ("dx",), ()):
        if n == 0 and names in (("dx",), ()):
            continue  # nothing to write
        grads = sum({"dx": 1, "dw": 2, "db": 4}[k] for k in names)
        need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], grads)
        ws, whole = guarded(need, 255)
        out, loss = outputs(c, names), torch.empty(n, device="cuda")
        capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, lse, **out, bias=c["bias"],
                            weight=c["weight"], workspace=ws)
        assert untouched(whole, need), (names, "one call")
        if n:
            check_all(dict(out, loss=loss), want)
        else:
            assert not any(v.any() for v in out.values())
        if not names:
            continue
        need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], grads, True)
        ws, whole = guarded(need, 255)
        capi.tb_linear_xent_grad(c["x"], c["w"], c["target"], lse, **out, bias=c["bias"],
                                 weight=c["weight"], workspace=ws)
        assert untouched(whole, need), (names, "gradients alone")


@pytest.mark.parametrize("dtype, n, D, C", [(BF16, 4096, 256, 16385), (F32, 2048, 128, 8193),
                                            (F32, 1500, 64, 4096 + 64), (BF16, 300, 64, 40001)])
def test_sums_in_parts_stay_in_their_place(dtype, n, D, C):
    """Tokens behind whole tiles whose dw is summed in parts."""
    from paper_2608_21343_amd import capi
    c = R.case(n, D, C, dtype, 2, device="cuda")
    want = R.expected(c)
    for names in (("dw",), ("dx", "dw", "db")):
        grads = sum({"dx": 1, "dw": 2, "db": 4}[k] for k in names)
        need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], grads)
        ws, whole = guarded(need, 255)
        out, loss = outputs(c, names), torch.empty(n, device="cuda")
        capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, None, **out, bias=c["bias"],
                            workspace=ws)
        assert untouched(whole, need)
        check_all(dict(out, loss=loss), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, D, C", [(70001, 8, 29), (70001, 8, 64), (70000, 8, 65), (9000, 70, 128),
                                     (70001, 8, 129), (9000, 70, 320), (9000, 70, 321),
                                     (1_600_000, 4, 64), (3000, 40, 1025), (300, 64, 50001)])
def test_few_tokens_and_many_rows(n, D, C, dtype):
    """Gradients in rows as long as the tokens need, in one piece and in several."""
    from paper_2608_21343_amd import capi
    c = R.case(n, D, C, dtype, 2, device="cuda", gaps=True)
    want = R.expected(c)
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7)
    ws, whole = guarded(need, 255)
    out, loss, lse = outputs(c), *torch.empty((2, n), device="cuda")
    capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, lse, **out, bias=c["bias"], workspace=ws)
    assert untouched(whole, need)
    check_all(dict(out, loss=loss), want)
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7, True)
    ws, whole = guarded(need, 255)
    capi.tb_linear_xent_grad(c["x"], c["w"], c["target"], lse, **out, bias=c["bias"], workspace=ws)
    assert untouched(whole, need)
    check_all(out, want)


@pytest.mark.parametrize("dtype, n", [(F32, 64), (F32, 65), (BF16, 32), (BF16, 1)])
def test_the_largest_vocabulary(dtype, n):
    """The most logits that few rows keep, and one row more."""
    from paper_2608_21343_amd import capi
    c = R.case(n, 16, 1 << 20, dtype, 2, device="cuda")
    want = R.expected(c)
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7)
    ws, whole = guarded(need, 255)
    out, loss, lse, low = outputs(c), *torch.empty((3, n), device="cuda")
    capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, lse, **out, bias=c["bias"],
                        out_low=low, workspace=ws)
    assert untouched(whole, need)
    check_all(dict(out, loss=loss), want)
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7, True)
    ws, whole = guarded(need, 255)
    capi.tb_linear_xent_grad(c["x"], c["w"], c["target"], lse, **out, bias=c["bias"],
                             lse_low=low, workspace=ws)
    assert untouched(whole, need)
    check_all(out, want)

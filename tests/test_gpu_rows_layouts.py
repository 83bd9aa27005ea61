"""Every layout of the row operators (waves a row, pieces a lane, rows whole or
cut) at the numbers of rows that take it, every row against float64. That the
cases take the layouts they are named after, and that these are all there are,
is checked without a GPU."""

import itertools

import pytest

from tests import rows_layouts as L


def _plan(dtype, C, n, grad):
    from paper_2608_21343_amd import capi
    waves, pieces, segments = capi.tb_debug_rows_plan(
        capi.TB_F32 if dtype == L.F32 else capi.TB_BF16, n, C, grad)
    return waves, pieces, segments > 1


@pytest.mark.parametrize("grad", [False, True])
def test_cases_take_their_layouts_and_all_of_them(grad):
    table = L.GRAD if grad else L.READ
    for dtype, layout, C, n in L.cases(table):
        assert _plan(dtype, C, n, grad) == layout, (dtype, C, n)
    widths = sorted({C + d for t in (L.READ, L.GRAD) for _, _, C, _ in L.cases(t)
                     for d in (-1, 0, 1)} | {2, 1 << 19, 1 << 20})
    numbers = sorted({n + d for t in (L.READ, L.GRAD) for _, _, _, n in L.cases(t)
                      for d in (-1, 0, 1)} | {1, 2, 127, 128, 2047, 2048, 4096, 1 << 20})
    for dtype in table:
        there = {_plan(dtype, C, n, grad) for C, n in itertools.product(widths, numbers)}
        assert there == set(table[dtype])


def test_plan_refusals():
    from paper_2608_21343_amd import capi
    for args in ((2, 1, 9), (0, 0, 9), (0, 1 << 41, 9), (0, 1, 1), (0, 1, (1 << 20) + 1)):
        with pytest.raises(capi.TbError):
            capi.tb_debug_rows_plan(*args)
    assert capi.LIB.tb_debug_rows_plan(0, 1, 9, 2, None) == capi.TB_EINVAL
    assert capi.LIB.tb_debug_rows_plan(0, 1, 9, 0, None) == capi.TB_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, layout, C, n", L.cases(L.READ), ids=L.name)
def test_scores(dtype, layout, C, n):
    L.check_scores(dtype, C, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, layout, C, n", L.cases(L.GRAD), ids=L.name)
def test_gradients(dtype, layout, C, n):
    L.check_grad(dtype, C, n)


@pytest.mark.gpu
@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("dtype, layout, C, n", L.cases(L.GRAD), ids=L.name)
def test_distillation(dtype, layout, C, n, tail):
    L.check_distill(dtype, C, n, tail)


@pytest.mark.gpu
@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("dtype, layout, C, n", L.cases(L.READ), ids=L.name)
def test_losses(dtype, layout, C, n, tail):
    L.check_distill(dtype, C, n, tail, grad=False)

"""The binding of the row operators on tensors of host memory: how it reads
shapes and strides (nothing is launched; a tensor's memory is never touched)."""

import pytest
import torch

from paper_2608_21343_amd import capi, rowops

V1 = 10


def _spread(*shape):
    """Logits of padded rows."""
    return torch.zeros(*shape, V1 + 3)[..., :V1]


def _last_place(x, rows, step):
    return x.storage_offset() + (rows - 1) * step + V1 - 1


# views whose rows are the same memory several times: inner, middle and outer
# dimensions, and several of them
EXPANDED = {
    "inner": torch.zeros(4, 1, V1).expand(4, 3, V1),
    "inner of one": torch.zeros(1, 1, V1).expand(1, 3, V1),
    "outer": torch.zeros(1, 3, V1).expand(4, 3, V1),
    "both": torch.zeros(1, 1, V1).expand(4, 3, V1),
    "first of four": torch.zeros(1, 4, 3, V1).expand(2, 4, 3, V1),
    "second of four": torch.zeros(2, 1, 3, V1).expand(2, 4, 3, V1),
    "third of four": torch.zeros(2, 4, 1, V1).expand(2, 4, 3, V1),
    "inner two of four": torch.zeros(2, 1, 1, V1).expand(2, 4, 3, V1),
    "outer two of four": torch.zeros(1, 1, 3, V1).expand(2, 4, 3, V1),
    "two dimensions": torch.zeros(1, V1).expand(3, V1),
    "padded": _spread(4, 1).expand(4, 3, V1),
    "between dimensions of one": torch.zeros(4, 1, 1, V1).expand(4, 3, 1, V1),
    "transposed": torch.zeros(4, 1, V1).expand(4, 3, V1).transpose(0, 1),
}


@pytest.mark.parametrize("name", EXPANDED)
def test_expanded_rows_are_refused_and_copied(name):
    x = EXPANDED[name]
    with pytest.raises(ValueError, match="overlap|evenly"):
        capi._rows(x)
    with pytest.raises(ValueError, match="grad rows"):
        capi._rows(x, "grad")
    y = rowops._even(x)
    assert y.is_contiguous() and y.shape == x.shape
    rows, width, step = capi._rows(y)
    assert rows * width == x.numel() and step == width


@pytest.mark.parametrize("x, want", [
    (torch.zeros(V1), (1, V1, V1)),
    (torch.zeros(3, V1), (3, V1, V1)),
    (torch.zeros(4, 3, V1), (12, V1, V1)),
    (torch.zeros(4, 1, 3, 1, V1), (12, V1, V1)),
    (_spread(4, 3), (12, V1, V1 + 3)),
    (_spread(2, 4, 3)[:, :1, :1], (2, V1, 12 * (V1 + 3))),
    (_spread(2, 4, 3)[:, :, 1], (8, V1, 3 * (V1 + 3))),
    (_spread(4, 3)[::2, 1], (2, V1, 6 * (V1 + 3))),
    # expanded, but only by dimensions of size 1
    (torch.zeros(4, 1, V1).expand(4, 1, V1), (4, V1, V1)),
    (torch.zeros(4, 3, V1).expand(1, 4, 3, V1), (12, V1, V1)),
])
def test_rows_of_views(x, want):
    assert capi._rows(x) == want
    assert _last_place(x, want[0], want[2]) < x.untyped_storage().nbytes() // 4
    assert rowops._even(x) is x


def test_rows_address_what_the_view_addresses():
    """Of views of every kind: accepted rows are those of the view, in order."""
    import itertools
    taken = 0
    for shape in itertools.product((1, 2, 3), repeat=3):
        for strides in itertools.product((0, 10, 13, 20, 30, 39, 60, 90), repeat=3):
            x = torch.empty(600).as_strided((*shape, V1), (*strides, 1))
            try:
                rows, width, step = capi._rows(x)
            except ValueError:
                continue
            want = [sum(i * s for i, s in zip(at, strides))
                    for at in itertools.product(*map(range, shape))]
            assert (rows, width) == (len(want), V1)
            assert want == [i * step for i in range(rows)] and (rows == 1 or step >= V1)
            taken += 1
    assert taken > 100


@pytest.mark.parametrize("shape", [(0, V1), (0, 3, V1), (2, 0, V1), (2, 3, 0, V1), (2, 0, 3, V1),
                                   (0, 0, V1)])
def test_no_rows_of_any_shape(shape):
    assert capi._rows(torch.zeros(shape)) == (0, V1, V1)
    assert capi._rows(torch.zeros(*shape[:-1], V1 + 3)[..., :V1]) == (0, V1, V1)
    assert rowops._even(torch.zeros(shape)).shape == shape


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(2, 0), (0, 3), (2, 0, 3)])
def test_calls_without_rows_of_any_shape(lead):
    z = torch.zeros(*lead, V1, device="cuda", requires_grad=True)
    tok = torch.zeros(*lead, 2, dtype=torch.int32, device="cuda")
    got = rowops.token_scores(z, tok, 3)
    assert got.logprob.shape == (*lead, 2) and got.alt.shape == (*lead, 3)
    loss = rowops.distill_loss(z, tok, torch.zeros(*lead, 2, device="cuda"))
    (loss.sum() + got.logprob.sum()).backward()
    assert loss.shape == lead and z.grad.shape == z.shape


LEAD = (4, 3)
TEACHERS = {
    "lists of transposed rows": dict(teacher_tok=(3, 4, 5), teacher_score=(3, 4, 5)),
    "flat lists": dict(teacher_tok=(12, 5), teacher_score=(12, 5)),
    "scores of another number": dict(teacher_score=(4, 3, 4)),
    "scores of transposed rows": dict(teacher_score=(3, 4, 5)),
    "transposed weights": dict(weight=(3, 4)),
    "flat weights": dict(weight=(12,)),
    "weights of one column": dict(weight=(4, 3, 1)),
    "one weight": dict(weight=()),
}


@pytest.mark.parametrize("entry", [rowops.distill_loss, rowops.distill_step])
@pytest.mark.parametrize("name", TEACHERS)
def test_teachers_of_other_shapes_are_refused(entry, name):
    """As many elements are not enough: they would be taken for other rows."""
    shape = {"teacher_tok": (4, 3, 5), "teacher_score": (4, 3, 5), "weight": (4, 3),
             **TEACHERS[name]}
    args = {k: torch.zeros(s, dtype=torch.int32 if k == "teacher_tok" else torch.float32)
            for k, s in shape.items()}
    with pytest.raises(ValueError, match="|".join(TEACHERS[name]) + " must"):
        entry(torch.zeros(*LEAD, V1), **args)


@pytest.mark.parametrize("entry", [rowops.distill_loss, rowops.distill_step])
def test_teachers_of_the_rows_shapes_are_taken(entry):
    """Up to the library, which takes device tensors only."""
    for lead in (LEAD, (6,), (), (2, 0)):
        tok = torch.zeros(*lead, 5, dtype=torch.int32)
        for weight in (None, torch.ones(lead)):
            with pytest.raises(ValueError, match="device"):
                entry(torch.zeros(*lead, V1), tok, torch.zeros(*lead, 5), weight=weight)


@pytest.mark.parametrize("n_alt", [0, 8, 64])
@pytest.mark.parametrize("dtype", [capi.TB_F32, capi.TB_BF16])
@pytest.mark.parametrize("width", [1025, 16388, 20000, 33000, 65540, 131073, 131080, 400003, 1 << 20])
def test_a_workspace_serves_fewer_rows(dtype, width, n_alt):
    """Bytes for n rows suffice for any call of up to n rows."""
    need = [capi.LIB.tb_rows_workspace_bytes(dtype, n, width, n_alt)
            for n in [*range(0, 2600), 4096, 8192, 1 << 20]]
    assert need == sorted(need)
    # cut where there are many rows: those that take more than four waves
    assert (need[-1] > 0) == (width > (16387 if dtype == capi.TB_F32 else 32775))
    # and those of fewer alternatives for any call of fewer
    if n_alt:
        for n in (1, 64, 65, 512, 513, 600, 4096):
            assert (capi.LIB.tb_rows_workspace_bytes(dtype, n, width, n_alt - 1)
                    <= capi.LIB.tb_rows_workspace_bytes(dtype, n, width, n_alt))


def test_workspace_of_a_tensor():
    """One row as a vector, and types that the operators do not take."""
    for dtype, code in ((torch.float32, capi.TB_F32), (torch.bfloat16, capi.TB_BF16)):
        x = torch.zeros(3, 400003, dtype=dtype)
        for t, n in ((x, 3), (x[0], 1), (x[:, None], 3)):
            want = capi.LIB.tb_rows_workspace_bytes(code, n, 400003, 5)
            assert capi.tb_rows_workspace_bytes(t, 5) == want > 0
        for other in (torch.float16, torch.float64, torch.int32):
            for t in (x.to(other), x[0].to(other)):
                with pytest.raises(ValueError, match="float32 or bfloat16"):
                    capi.tb_rows_workspace_bytes(t, 5)


def test_workspace_of_arguments_out_of_range():
    for width, n_alt, word in ((9, 65, "n_alt"), (9, -1, "n_alt"), ((1 << 20) + 1, 0, "v_plus")):
        with pytest.raises(capi.TbError, match=word):
            capi.tb_rows_workspace_bytes(torch.zeros(1, width), n_alt)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, width", [(torch.bfloat16, 131073), (torch.float32, 70001)])
def test_one_workspace_for_several_numbers_of_rows(dtype, width):
    """Made for the largest batch and used for smaller ones, whose cuts differ."""
    g = torch.Generator(device="cuda").manual_seed(width)
    z = torch.randn(600, width, generator=g, device="cuda").to(dtype)
    work = torch.empty(capi.tb_rows_workspace_bytes(z, 8), dtype=torch.uint8, device="cuda")
    alt = torch.empty(600, 8, dtype=torch.int32, device="cuda")
    alt_lp = torch.empty(600, 8, device="cuda")
    want = torch.topk(z[:512].float(), 8, dim=1).values
    for n in (600, 513, 512, 64, 1):
        grad, loss = torch.empty_like(z[:n]), torch.empty(n, device="cuda")
        capi.tb_token_logprobs(z[:n], out_alt=alt[:n], out_alt_logprob=alt_lp[:n], workspace=work)
        capi.tb_distill(z[:n], alt[:n], alt_lp[:n], loss, grad, tail=True, workspace=work)
        m = min(n, 512)
        # ids of the largest values; equal values in either order
        got = torch.gather(z[:m].float(), 1, alt[:m].long())
        assert bool((got == want[:m]).all())
        assert float(loss.abs().max()) < 3e-5  # a student equal to its teacher
        assert float(grad.float().abs().max()) < 3e-5

"""The output layer's cross entropy on the GPU against float64 where its launches
differ: tiles of 256, 128 and 64, tokens behind whole tiles, pieces of the vocabulary,
sums in parts, few rows read where they are, logits kept or made again."""

import math

import pytest
import torch

from tests import linear_reference as R
from tests.test_gpu_linear import check_all, grad, step

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

TILES = [  # rows, width, V + 1
    (16000, 512, 1025), (16000, 64, 1024), (4096, 192, 16385), (4100, 64, 16384 + 37),
    (4096, 64, 16384 + 64), (4096, 64, 16384 + 65), (600, 128, 8193), (2047, 256, 4097),
    (2049, 256, 4097), (20000, 64, 70), (100, 64, 40001), (257, 1024, 513), (513, 100, 2304),
    (1000, 2100, 300), (66, 4100, 129),
]
FEW = [  # up to 64 rows, of both sides of 65,536 tokens
    (1, 72, 300), (16, 64, 65536), (17, 40, 65537), (32, 520, 1025), (33, 64, 70001),
    (48, 256, 300), (64, 1024, 8193), (1, 2048, 131073), (64, 8, 66000),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, D, C", TILES + FEW)
def test_in_one_call_and_in_two(n, D, C, dtype):
    some = (n + C) % 2 == 0
    c = R.case(n, D, C, dtype, n + D, bias=C % 4 != 0, weighted=some, gaps=some, device="cuda")
    want = R.expected(c)
    got = step(c)
    check_all(got, want)
    check_all(step(c, ()), {k: want[k] for k in ("loss", "lse")})
    one = torch.ones(n, device="cuda")
    check_all(grad(c, got["lse"], one, None), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, C", [(6000, 45057), (3000, 60 * 1024 + 3)])
def test_pieces_with_tokens_behind_them(n, C, dtype):
    c = R.case(n, 64, C, dtype, 5, device="cuda", gaps=True)
    want = R.expected(c)
    got = step(c)
    check_all(got, want)
    check_all(grad(c, got["lse"], torch.ones(n, device="cuda"), None), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, D, C", [(1500, 256, 1025), (16000, 64, 1025), (100, 64, 40001),
                                     (5000, 64, 45057), (20000, 64, 70), (40, 64, 70001),
                                     (64, 100, 513), (3, 64, 300)])
def test_whatever_the_workspace_holds(n, D, C, dtype):
    from paper_2608_21343_amd import capi
    c = R.case(n, D, C, dtype, 12, device="cuda", weighted=True, gaps=True)
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        got = step(c, workspace=ws)
        first = first or got
        for name in first:
            assert bool((first[name] == got[name]).all()), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [64, 65, 3000])
def test_targets_at_the_edges_of_tiles(n, dtype):
    """Every token of the first and last tiles as a target, each once or more."""
    D, C = 64, 8192 + 1
    c = R.case(n, D, C, dtype, 9, device="cuda")
    edges = [0, 63, 64, 127, 128, 255, 256, 257, 4095, 4096, 8063, 8064, 8127, 8128, 8191, 8192]
    c["target"] = torch.tensor([edges[i % len(edges)] for i in range(n)], dtype=torch.int32,
                               device="cuda")
    check_all(step(c), R.expected(c))


def test_rows_far_apart():
    """Weights whose rows lie 2^23 values apart."""
    n, D, C, far = 100, 64, 258, (1 << 23) + 64
    c = R.case(n, D, C, BF16, 4, device="cuda")
    buf = torch.empty(C * far, dtype=BF16, device="cuda")
    w = buf.as_strided((C, D), (far, 1))
    w.copy_(c["w"])
    c["w"] = w
    want = R.expected(c)
    from paper_2608_21343_amd import capi
    loss, dw = torch.empty(n, device="cuda"), torch.empty((C, D), dtype=BF16, device="cuda")
    dx = torch.empty((n, D), dtype=BF16, device="cuda")
    capi.tb_linear_xent(c["x"], w, c["target"], loss, None, dx=dx, dw=dw, bias=c["bias"])
    check_all({"loss": loss, "dx": dx, "dw": dw}, want)


@pytest.mark.parametrize("n", [40, 300])
def test_tokens_without_weights(n):
    """float32: tokens without weights beside others, and weights of very different sizes."""
    c = R.case(n, 96, 700, F32, 8, device="cuda")
    c["w"][::3] = 0.0
    c["w"][1::3] *= 2.0 ** -40
    check_all(step(c), R.expected(c))
    c["w"][:] = 0.0
    check_all(step(c), R.expected(c))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 300])
@pytest.mark.parametrize("mask", [-math.inf, -3e38])
def test_masked_tokens_hold_anything_finite(mask, n, dtype):
    """Weights of tokens that the bias masks, however large, change nothing."""
    c = R.case(n, 96, 700, dtype, 8, device="cuda")
    c["bias"][7::50] = mask
    c["target"][c["target"] % 50 == 7] = 1
    c["w"][7::50] = 0.0
    want = R.expected(c)
    check_all(step(c), want)
    for value in (1e30, -1e30):
        # (x stays below 8: what they add leaves a mask of -3e38 far below the others)
        c["w"][7::50] = value
        check_all(step(c), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [9, 40, 300])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_masked_tokens_that_are_not_finite(value, n, dtype):
    """A mask does not hide a NaN: -inf and it, or an infinity of the other sign, are NaN."""
    c = R.case(n, 96, 700, dtype, 8, device="cuda")
    c["bias"][7] = -math.inf
    c["target"][c["target"] == 7] = 1
    c["w"][7] = value
    z = c["x"].double() @ c["w"].double().t() + c["bias"].double()
    bad = torch.isnan(z).any(1)
    assert bool(bad.any())
    for got in (step(c), step(c, ())):
        assert bool((torch.isnan(got["loss"]) == bad).all())
        assert bool((torch.isnan(got["lse"]) == bad).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [9, 40, 300])
def test_every_token_masked_by_a_number(n, dtype):
    """Logits that are all the same number near the type's lowest: loss log(V+1), and
    gradients without a NaN."""
    D, C = 96, 700
    c = R.case(n, D, C, dtype, 8, device="cuda")
    c["x"][:] = 0.0
    c["bias"][:] = -3.0e38
    want = math.log(C)
    got = step(c)
    two = grad(c, got["lse"], torch.ones(n, device="cuda"), None)
    # 700 exponentials of 0 are exact, and so is their sum; the logarithm to two steps
    assert float((got["loss"].double() - want).abs().max()) <= 4 * 2.0 ** -24 * want
    assert bool((got["lse"].double() + 3.0e38 <= 2.0 ** -8 * 3.0e38).all())
    for out in (got, two):
        for name in ("dx", "dw", "db"):
            assert bool(torch.isfinite(out[name]).all()), name


@pytest.mark.parametrize("n, D, C", [(1, 64, 300), (2, 127, 339), (16, 512, 1025), (17, 40, 65537),
                                     (31, 320, 999), (32, 64, 70001)])
def test_gradients_of_few_bfloat16_rows(n, D, C):
    """Calls of up to 32 rows keep what rounding the logits' gradients left: 2^-16 of them is
    lost and not 2^-8."""
    some = n % 2 == 0
    c = R.case(n, D, C, BF16, n + D, weighted=some, gaps=some, device="cuda")
    weight = None if c["weight"] is None else c["weight"].double()
    x = torch.where((c["target"] != -1)[:, None], c["x"].double(), 0.0)
    w = c["w"].double()
    _, lse, z = R.forward(x, w, c["target"], c["bias"].double(), weight)
    G = R.logit_grad(z, lse, c["target"], weight).abs()
    rounded = R.U[BF16] - 2.0 ** -16
    want = R.expected(c)
    for name, size in (("dx", G @ w.abs()), ("dw", G.t() @ x.abs())):
        value, tol = want[name]
        want[name] = (value, tol - rounded * size)
    got = step(c)
    check_all(got, want)
    check_all(grad(c, got["lse"], torch.ones(n, device="cuda"), None), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 2, 300, 3000])
def test_one_gradient_for_all_rows(n, dtype):
    """A loss gradient that is one value, expanded: the same bits as one a row."""
    c = R.case(n, 64, 300, dtype, 7, device="cuda", gaps=True)
    lse = step(c, ())["lse"]
    one = torch.full((1,), 0.75, device="cuda")
    for name, value in grad(c, lse, one.expand(n), None).items():
        again = grad(c, lse, one.repeat(n), None)[name]
        assert bool((value == again).all()), name


def test_two_calls_at_once():
    cases = [R.case(n, 256, C, dtype, 2, device="cuda", gaps=True)
             for n, C, dtype in ((900, 4097, BF16), (700, 3001, F32))]
    want = [step(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                got.append(step(c))
        torch.cuda.synchronize()
        for one, right in zip(got, want):
            for name in right:
                assert bool((one[name] == right[name]).all()), name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_losses_of_large_logits(dtype):
    """The loss keeps its digits where lse and the target's logit are large and near."""
    D, C = 64, 600
    for n in (70, 20):
        c = R.case(n, D, C, dtype, 3, device="cuda", bias=False)
        c["x"][:] = 0.0
        c["x"][:, 0] = 1.0
        c["w"][:] = 1016.0
        c["w"][5] = 1024.0
        c["target"][:] = 5
        loss = step(c, ())["loss"].double()
        right = math.log1p((C - 1) * math.exp(-8.0))
        # logits and their differences are exact; 80 additions above 1, half a step each; an
        # exponential's argument below 16 in units of log 2 (2^-21) and log 2's own rounding
        # (2^-20), its function and the logarithm (2^-22). Half a step of lse is 2^-14.
        assert float((loss - right).abs().max()) <= 80 * 2.0 ** -24 + right * 2.0 ** -19


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [9, 20, 70])
def test_gradients_of_certain_rows(n, dtype):
    """p - 1 keeps its digits where lse is large and p near 1, in one call and in two."""
    from paper_2608_21343_amd import capi
    D, C = 64, 600
    c = R.case(n, D, C, dtype, 3, device="cuda", bias=False)
    c["x"][:] = 0.0
    c["x"][:, 0] = 1.0
    c["w"][:] = 1008.0
    c["w"][5] = 1024.0
    c["target"][:] = 5
    p = math.exp(-16.0) / (1 + (C - 1) * math.exp(-16.0))
    want = torch.full((C,), p * n, dtype=torch.float64, device="cuda")
    want[5] = -p * (C - 1) * n
    # 1 / sum (or the exponential of lse's rest) and a times it: four roundings of half a step
    # near 1 and as many of the sum of 64 tokens or fewer near 1; exponentials of -16 to 2^-19
    # of themselves; n additions; the result's own rounding
    tol = R.U[dtype] * want.abs() + 2.0 ** -18 * want.abs() + (n + 4) * 2.0 ** -24 * want.abs()
    tol[5] += n * (4 + 68) * 2.0 ** -24
    loss, lse, low = torch.empty((3, n), device="cuda")
    out = {k: torch.empty(C, dtype=dtype, device="cuda") for k in ("one", "two")}
    capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, lse, db=out["one"], out_low=low)
    capi.tb_linear_xent_grad(c["x"], c["w"], c["target"], lse, db=out["two"], lse_low=low)
    for name, db in out.items():
        assert bool(((db.double() - want).abs() <= tol).all()), name
    exact = 1024.0 + math.log1p((C - 1) * math.exp(-16.0))
    assert float((lse.double() + low.double() - exact).abs().max()) <= 72 * 2.0 ** -24
    assert float(low.abs().max()) <= 2.0 ** -14  # half a step of lse

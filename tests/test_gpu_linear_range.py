"""The output layer's float32 units: features, weights and gradients of sizes whose
products are ordinary numbers, while those of their units are not."""

import pytest
import torch

from tests import linear_reference as R
from tests.test_gpu_linear import check_all, grad, step

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.mark.parametrize("n", [70, 300, 2000])
@pytest.mark.parametrize("power", [112, 108, -108])
def test_large_weights_and_small_features(power, n):
    """Logits of order 1, 2^28 times the units of their factors; the other way round, too."""
    c = R.case(n, 64, 520, F32, 4, device="cuda", gaps=True)
    c["w"] *= 2.0 ** power
    c["x"] *= 2.0 ** -power
    want = R.expected(c)
    got = step(c)
    check_all(got, want)
    check_all(step(c, ()), {k: want[k] for k in ("loss", "lse")})
    check_all(grad(c, got["lse"], torch.ones(n, device="cuda"), None), want)


@pytest.mark.parametrize("n", [70, 300])
@pytest.mark.parametrize("size", [2.0 ** 60, 2.0 ** -60])
def test_large_and_small_gradients(size, n):
    """Weights of the rows and of the layer that are both large, or both small: dx is their
    product, dw that of the rows' weights and the features."""
    c = R.case(n, 64, 520, F32, 4, device="cuda", weighted=True)
    c["w"] *= size
    c["x"] *= 1 / size
    c["weight"] *= size
    want = R.expected(c)
    got = step(c)
    check_all(got, want)
    check_all(grad(c, got["lse"], torch.ones(n, device="cuda"), None), want)


@pytest.mark.parametrize("n", [70, 300])
def test_logits_of_a_million(n):
    """Of weights near float32's end and features 2^-97 times an ordinary size."""
    c = R.case(n, 64, 520, F32, 4, device="cuda")
    c["w"] *= 2.0 ** 117
    c["x"] *= 2.0 ** -97
    want = R.expected(c)
    got = step(c, ())
    check_all(got, {k: want[k] for k in ("loss", "lse")})
    assert bool(torch.isfinite(got["loss"]).all())


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16])
@pytest.mark.parametrize("n", [9, 40, 300])
def test_lse_of_tokens_that_are_all_masked_by_a_number(n, dtype):
    """It is that number, from either side, alone and beside gradients."""
    c = R.case(n, 96, 700, dtype, 8, device="cuda")
    c["x"][:] = 0.0
    c["bias"][:] = -3.0e38
    want = c["bias"][0].double()
    for got in (step(c), step(c, ())):
        # (log 700 is far below half a step of it)
        assert float((got["lse"].double() - want).abs().max()) <= 2.0 ** -24 * float(want.abs())

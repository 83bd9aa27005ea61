"""The workspace of the output layer's calls: how a call is laid out is decided on the
host, so no GPU is needed to ask for every size."""

import itertools

import pytest

P = 1 << 20  # an aligned address that nothing reads
F32, BF16 = 0, 1


def need(dtype, n, D, C, grads, with_lse=0, w=P, stride=None):
    from paper_2608_21343_amd import capi
    return capi.LIB.tb_linear_xent_workspace_bytes(dtype, n, D, C, w, stride or D, grads, with_lse)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_size_has_a_plan(dtype):
    """Few tokens with millions of rows, whose gradients take more than one piece, among them."""
    tokens = [*range(2, 70), 127, 128, 129, 255, 256, 257, 300, 319, 320, 321, 383, 384, 385, 511,
              512, 513, 576, 577, 1025, 4097, 32769, 131073, (1 << 20) - 255, 1 << 20]
    rows = [0, 1, 2, 17, 33, 64, 65, 257, 4096, 70001, 350_000, 400_000, 800_000, 1_600_000,
            3_500_000, 1 << 23, 1 << 24]
    for C, n, D in itertools.product(tokens, rows, (1, 64, 513)):
        for grads, with_lse in itertools.product((0, 1, 2, 4, 7), (0, 1)):
            assert need(dtype, n, D, C, grads, with_lse) > 0, (n, D, C, grads, with_lse)


def test_calls_without_rows_need_no_output():
    """The binding passes NULL for an output of no values."""
    from paper_2608_21343_amd import capi
    assert capi.LIB.tb_linear_xent(0, 2 * P, 0, 1, 0, 64, 100, 64, 64, 0, 0, 0, 0, 0, 0, 64, 0, 64,
                                   0, 0, 0, 0) == 0
    assert capi.LIB.tb_linear_xent_grad(0, 2 * P, 0, 1, 0, 64, 100, 64, 64, 0, 0, 0, 0, 0, 1, 0, 0,
                                        64, 0, 64, 0, 0, 0, 0) == 0


@pytest.mark.parametrize("dtype, n, D, tokens", [
    (BF16, 4096, 2048, 131072), (F32, 2048, 1024, 32768), (BF16, 16384, 1024, 8192),
    (F32, 16000, 512, 1024)])
@pytest.mark.parametrize("grads", [2, 3, 7])
def test_a_token_behind_whole_tiles_takes_little(grads, dtype, n, D, tokens):
    """The blank, one more than a multiple of 256: the copy of a token's weights, its parts of dw
    (64 tokens in up to 64 parts), its gradients and their sums for every row."""
    for with_lse in (0, 1):
        even, odd = (need(dtype, n, D, C, grads, with_lse) for C in (tokens, tokens + 1))
        assert odd <= even + 64 * 64 * D * 4 + 2 * 256 * n * 4 + (2 << 20)

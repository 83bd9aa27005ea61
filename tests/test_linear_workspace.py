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


def up(x, m):
    return -(-x // m) * m


def most(dtype, n, D, C, grads, with_lse):
    """What a call may ask for: 16-bit planes of features and weights, statistics of every row and
    64 tokens, logits of up to 256 MB, gradients of logits of 384 MB or of a piece of 256 tokens
    and 64 behind them in whole tiles, their sums for every 16 rows, sums in parts, and some
    words a row."""
    planes, np, dp = 2 - dtype, up(n, 256), up(D, 64)
    size = 64 * np + 4 * 256 + (n >> 8) * 8 + 20 * 256
    size += planes * np * dp * 2 * (2 if dtype == F32 and grads & 2 else 1) + planes * C * dp * 2
    size += n * max(2 * (C // 64 + 2), min(C // 16 + 1, 4096)) * 8
    if grads:
        columns = up(C, 64) if C <= 128 else up(min(C, 320), 256)
        G = max(384 << 20, planes * np * 2 * columns)
        size += G + (0 if with_lse and n > 64 else 256 << 20)
        size += G // 8 if grads & 4 else 0
        size += 2 * n * dp * 4 + (256 << 20) if grads & 1 else 0
        size += 256 << 20 if grads & 2 else 0
    return size


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_workspaces_are_bounded(dtype):
    """Whatever the numbers of rows and tokens are, one large and the other small among them."""
    tokens = [2, 50, 64, 65, 128, 257, 300, 1024, 1025, 4097, 32769, 131073, 700_000, 1 << 20]
    rows = [1, 16, 17, 33, 64, 65, 257, 4096, 70001, 400_000, 1 << 20, 3_100_000, 1 << 24]
    for C, n, D in itertools.product(tokens, rows, (1, 64, 513, 2048)):
        for grads, with_lse in itertools.product((0, 1, 2, 4, 7), (0, 1)):
            got, bound = need(dtype, n, D, C, grads, with_lse), most(dtype, n, D, C, grads, with_lse)
            assert got <= bound, (n, D, C, grads, with_lse, got / bound)


@pytest.mark.parametrize("dtype, n, D, C, grads, bytes_", [
    (F32, 1 << 20, 1, 50, 4, 0.9e9), (BF16, 3_100_000, 64, 64, 4, 1.0e9),
    (BF16, 1, 64, 700_000, 7, 0.1e9)])
def test_workspaces_of_few_tokens_or_rows(dtype, n, D, C, grads, bytes_):
    """Rows and tokens that are not there take no room."""
    assert need(dtype, n, D, C, grads) <= bytes_

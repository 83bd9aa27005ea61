"""Row operators on the GPU against their float64 forms (tests/rows_reference.py).

Tolerances follow from float32 arithmetic, eps = 2^-24 (half a step): an
exponent x = (z - max) / tau carries at most 3 roundings (the scaled constant,
the product, the difference), so that 2^t is off by 3 eps |x| and 2 eps of the
exponential itself; a sum of such terms by their mean, 3 eps E|x| + 2 eps, and
the roundings of adding them up, at most 24 on the way from a lane to the row.
With |x| and E|x| up to 40 in these inputs: log-sum-exp and log probabilities
within SUM = 160 eps = 1e-5 (and 4 eps of a value's own size), an entropy's dot
product of terms x 2^t within another factor |x| of that in its tail, 3e-5, a
gradient within 1e-5 of the magnitudes that it is made of; bfloat16 gradients
are off by their one rounding, 2^-8 of the value (half a step of 2^-7), too. With the tail, q_rest =
1 - sum q is off by 16 eps = 1e-6 absolutely, which counts by log(q_rest /
p_rest) + 1 in the loss and by 1 / p_rest in the gradient."""

import math

import numpy as np
import pytest
import torch

from tests import rows_reference as R

pytestmark = pytest.mark.gpu

SUM = 1e-5
REL = 3e-7
NEG = -math.inf
F32, BF16 = torch.float32, torch.bfloat16

# on both sides of every number of values that a wave's or workgroup's
# registers hold, and beyond all of them
EDGES = {F32: [2, 3, 4, 5, 63, 64, 257, 259, 260, 515, 516, 1025, 1027, 1028, 2051, 2052, 4099,
               4100, 8193, 8195, 8196, 16387, 16388, 32771, 32772, 65539, 65540, 131073, 400003],
         BF16: [2, 3, 7, 8, 9, 64, 257, 519, 520, 1025, 1031, 1032, 2055, 2056, 4103, 4104, 8193,
                8199, 8200, 16391, 16392, 32775, 32776, 65543, 65544, 131079, 131080, 400003]}
WIDTHS = [(d, c) for d in (F32, BF16) for c in EDGES[d]]


def ids(p):
    return {F32: "f32", BF16: "bf16"}.get(p, str(p)) if not isinstance(p, tuple) else \
        "-".join(ids(x) for x in p)


def make(seed, n, C, dtype, pad=0, std=2.0):
    """Rows with one clearly preferred token each, in a padded buffer."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((n, C), generator=g) * std
    z[torch.arange(n), torch.randint(0, C, (n,), generator=g)] += 6.0
    buf = torch.full((n, C + pad), 1e30, dtype=dtype)
    buf[:, :C] = z
    return buf.cuda()[:, :C], g


def host(z):
    return z.float().cpu().numpy()


def score(z, tokens, M, tau=1.0, lse=True, ent=True):
    from paper_2608_21343_amd import capi
    n, J = tokens.shape
    lp = torch.full((n, J), 77.0, device="cuda")
    o_lse = torch.full((n,), 77.0, device="cuda") if lse else None
    o_ent = torch.full((n,), 77.0, device="cuda") if ent else None
    alt = torch.full((n, M), 77, dtype=torch.int32, device="cuda") if M else None
    alt_lp = torch.full((n, M), 77.0, device="cuda") if M else None
    capi.tb_token_logprobs(z, tokens.cuda() if J else None, lp if J else None, o_lse, o_ent, alt,
                           alt_lp, temperature=tau)
    torch.cuda.synchronize()
    return tuple(None if x is None else x.cpu().numpy() for x in (lp, o_lse, o_ent, alt, alt_lp))


def close(got, want, abs_tol, rel=REL):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        ok = same | (np.abs(got - want) <= abs_tol + rel * np.abs(want))
    assert ok.all(), (np.argwhere(~ok)[:3].tolist(), got[~ok][:3], want[~ok][:3])


def check_scores(z, tokens, M, tau=1.0):
    got = score(z, tokens, M, tau)
    want = R.scores(host(z), tau, tokens.numpy(), M)
    close(got[0], want[0], SUM)
    close(got[1], want[1], SUM)
    close(got[2], want[2], 3e-5)
    if M:
        np.testing.assert_array_equal(got[3], want[3])
        close(got[4], want[4], SUM)


def given(g, n, C, J):
    t = torch.randint(0, C, (n, J), generator=g, dtype=torch.int32)
    if J > 1:
        t[0, 1] = t[0, 0]
        t[-1, -1] = -1
    return t


@pytest.mark.parametrize("dtype, C", WIDTHS, ids=ids)
def test_scores_at_every_width(dtype, C):
    n = 7 if C < 40000 else 2
    z, g = make(C, n, C, dtype, pad=3)
    for J, M in ((1, 8), (3, 0), (0, 1), (2, 64 if C < 140000 else 20)):
        check_scores(z, given(g, n, C, J), M)


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("dtype, C", [(F32, 50), (F32, 1025), (BF16, 1025), (F32, 5000),
                                      (BF16, 20000), (BF16, 150000)], ids=ids)
def test_every_number_of_alternatives(dtype, C, M):
    z, g = make(M, 5, C, dtype)
    check_scores(z, given(g, 5, C, 1), M)


@pytest.mark.parametrize("tau", [1e-4, 0.3, 1.7, 40.0, 1e4])
@pytest.mark.parametrize("dtype, C", [(F32, 1025), (BF16, 9001), (F32, 80001)], ids=ids)
def test_temperatures(dtype, C, tau):
    z, g = make(3, 4, C, dtype)
    got = score(z, given(g, 4, C, 2), 5, tau)
    tok = given(torch.Generator().manual_seed(0), 4, C, 2)
    got = score(z, tok, 5, tau)
    want = R.scores(host(z), tau, tok.numpy(), 5)
    # an exponent's error goes with its size
    size = max(1.0, float(np.abs(host(z)).max()) / tau)
    close(got[0], want[0], SUM, 6e-7)
    close(got[1], want[1], SUM, 6e-7)
    close(got[2], want[2], 3e-5)
    np.testing.assert_array_equal(got[3], want[3])
    close(got[4], want[4], SUM + 1e-7 * size, 6e-7)


def special_rows(C, dtype):
    """Rows where sums and selections go wrong, as float32 values of the type."""
    low = torch.finfo(dtype).min
    rows = []

    def row(fill):
        r = torch.full((C,), fill)
        rows.append(r)
        return r

    row(NEG)                                     # empty
    row(low)                                     # every token at the lowest value
    row(0.0)                                     # all alike
    r = row(NEG); r[C // 2] = 1.5                # one token
    r = row(NEG); r[[0, C - 1]] = torch.tensor([2.0, 2.0])
    r = row(low); r[[1, C // 3, C - 2]] = torch.tensor([0.5, -1.0, 3.0])
    r = row(-1e4); r[[0, C // 2]] = torch.tensor([1.0, 2.0])
    r = row(-1e30); r[C - 1] = -1e30
    r = row(1e30); r[0] = 1.5e30
    r = row(0.0); r[::2] = -0.0                  # both zeros are equal
    r = row(5.0); r[C // 4:] = torch.arange(C - C // 4).remainder(3).float()
    rows.append(torch.arange(C, 0, -1).float() * 0.01)   # descending
    rows.append(torch.arange(C).float() * 0.01)          # ascending
    rows.append(torch.linspace(-3, 3, C) + 1000.0)       # far from zero
    r = row(0.0); r[C // 2] = math.nan
    r = row(0.0); r[C // 2] = math.inf
    r = row(math.nan)
    r = row(NEG); r[0] = math.nan
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("M", [4, 40])
@pytest.mark.parametrize("dtype, C", [(F32, 9), (F32, 300), (F32, 1025), (BF16, 1025),
                                      (F32, 2100), (BF16, 8193), (F32, 20000), (BF16, 70001),
                                      (BF16, 140001), (F32, 70001)], ids=ids)
def test_special_rows(dtype, C, M):
    z = special_rows(C, dtype).cuda()
    n = z.shape[0]
    tok = torch.tensor([[0, C // 2, C - 1, -1]] * n, dtype=torch.int32)
    got = score(z, tok, M)
    want = R.scores(host(z), 1.0, tok.numpy(), M)
    # log probabilities of tokens at the lowest value are of that size
    close(got[0], want[0], SUM, 2e-7)
    close(got[1], want[1], SUM, 2e-7)
    close(got[2], want[2], 3e-5)
    np.testing.assert_array_equal(got[3], want[3])
    close(got[4], want[4], SUM, 2e-7)


@pytest.mark.parametrize("dtype, C", [(F32, 1025), (BF16, 5000), (F32, 100001)], ids=ids)
def test_tokens_out_of_range(dtype, C):
    z, g = make(4, 3, C, dtype)
    tok = torch.tensor([[0, -1, C], [-2, 1, 2**31 - 1], [C - 1, -2**31, 5]], dtype=torch.int32)
    check_scores(z, tok, 3)


@pytest.mark.parametrize("dtype, C", [(F32, 1025), (BF16, 1025), (BF16, 9000), (F32, 70000)],
                         ids=ids)
def test_ties_go_to_the_lowest_token(dtype, C):
    g = torch.Generator().manual_seed(C)
    z = (torch.randint(0, 4, (6, C), generator=g).float() * 0.5).to(dtype).cuda()
    check_scores(z, given(g, 6, C, 1), 64)


def test_optional_outputs_and_shapes():
    from paper_2608_21343_amd import capi
    z, g = make(5, 6, 301, F32, pad=7)
    tok = given(g, 6, 301, 2)
    full = score(z, tok, 5)
    part = score(z, tok, 0, lse=False, ent=False)
    np.testing.assert_array_equal(full[0], part[0])
    # [T, B, K, V+1] logits with padded rows and lists of the same leading shape
    z4 = z.unflatten(0, (3, 2, 1))
    lp = torch.empty((3, 2, 1, 2), device="cuda")
    capi.tb_token_logprobs(z4, tok.cuda().view(3, 2, 1, 2), lp)
    np.testing.assert_array_equal(lp.cpu().numpy().reshape(6, 2), full[0])
    # one row, given as a vector
    lp = torch.empty(2, device="cuda")
    capi.tb_token_logprobs(z[4], tok[4].cuda(), lp)
    np.testing.assert_array_equal(lp.cpu().numpy(), full[0][4])


# ---------------------------------------------------------------------------
# gradients


def run_grad(z, tok, d_lp, d_lse, d_ent, tau=1.0, in_place=False):
    from paper_2608_21343_amd import capi
    if in_place:
        buf = torch.full((z.shape[0], z.shape[1] + 3), 55.0, dtype=z.dtype, device="cuda")
        out = buf[:, :z.shape[1]]
        out.copy_(z)
        src = out
    else:
        buf = torch.full((z.shape[0], z.shape[1] + 3), 55.0, dtype=z.dtype, device="cuda")
        out, src = buf[:, :z.shape[1]], z

    def dev(x):
        return None if x is None else torch.tensor(x, dtype=F32).cuda()

    J = tok.shape[1]
    capi.tb_token_logprobs_grad(src, tok.cuda() if J else None, dev(d_lp) if J else None, out,
                                d_lse=dev(d_lse), d_entropy=dev(d_ent), temperature=tau)
    torch.cuda.synchronize()
    assert bool((buf[:, z.shape[1]:] == 55.0).all())  # nothing between rows is written
    return out.float().cpu().numpy()


def grad_size(z, tau, tok, d_lp, d_lse, d_ent):
    """The magnitudes that a gradient is made of."""
    n, C = z.shape
    size = np.zeros((n, C))
    for i in range(n):
        logp, lse = R.softmax_row(z[i], tau)
        if not lse > NEG:
            continue
        a = abs(d_lse[i]) if d_lse is not None else 0.0
        a += np.abs(d_lp[i]).sum()
        h = abs(d_ent[i]) if d_ent is not None else 0.0
        p = np.exp(logp)
        size[i] = p * (a + h * (np.abs(np.where(p > 0, logp, 0)) + R.entropy_row(logp)))
        for t, g in zip(tok[i], d_lp[i]):
            if 0 <= t < C:
                size[i, t] += abs(g)
    return size / tau


def check_grad(z, tok, seed=0, lse=True, ent=True, tau=1.0, in_place=False):
    n, J = tok.shape
    rng = np.random.default_rng(seed)
    d_lp = rng.normal(size=(n, J)).astype(np.float32)
    d_lse = rng.normal(size=n).astype(np.float32) if lse else None
    d_ent = rng.normal(size=n).astype(np.float32) if ent else None
    got = run_grad(z, tok, d_lp, d_lse, d_ent, tau, in_place)
    zh = host(z)
    want = R.score_grad(zh, tau, tok.numpy(), d_lp, d_lse, d_ent)
    size = grad_size(zh, tau, tok.numpy(), d_lp, d_lse, d_ent)
    close(got, want, 1e-5 * size + 1e-37, 2.0 ** -7.99 if z.dtype == BF16 else REL)
    return want


@pytest.mark.parametrize("dtype, C", WIDTHS, ids=ids)
def test_gradients_at_every_width(dtype, C):
    n = 6 if C < 40000 else 2
    z, g = make(C, n, C, dtype, pad=5)
    for J, lse, ent in ((1, False, False), (2, False, True), (0, True, False), (5, True, True)):
        check_grad(z, given(g, n, C, J), C, lse, ent, in_place=J == 5)


@pytest.mark.parametrize("J", [1, 2, 3, 4, 5, 33, 64])
@pytest.mark.parametrize("dtype, C", [(F32, 40), (BF16, 1025), (F32, 9000), (BF16, 140000)],
                         ids=ids)
def test_gradients_of_lists(dtype, C, J):
    """Lists of every length, with tokens listed twice and unused places."""
    z, g = make(J, 5, C, dtype)
    tok = given(g, 5, C, J)
    tok[1] = tok[1, 0]
    tok[2, ::2] = -1
    tok[3] = -1
    for in_place in (False, True):
        check_grad(z, tok, J, False, False, 1.9, in_place)
        check_grad(z, tok, J, True, True, 0.6, in_place)


@pytest.mark.parametrize("dtype, C", [(F32, 9), (F32, 1025), (BF16, 1025), (BF16, 8193),
                                      (F32, 20000), (F32, 70001)], ids=ids)
def test_gradients_of_special_rows(dtype, C):
    z = special_rows(C, dtype).cuda()
    tok = torch.tensor([[0, C // 2, C - 1]] * z.shape[0], dtype=torch.int32)
    check_grad(z, tok, 1, False, False)
    check_grad(z, tok, 2, True, True)


def test_gradient_of_nothing_and_of_bad_tokens():
    z = special_rows(1025, F32).cuda()
    n = z.shape[0]
    tok = torch.tensor([[3, -1]] * n, dtype=torch.int32)
    zero = np.zeros((n, 2), np.float32)
    got = run_grad(z, tok, zero, np.zeros(n), np.zeros(n))
    assert (got == 0).all()  # rows of NaN as well
    tok[2, 1] = 1025
    got = run_grad(z, tok, zero, None, None)
    assert np.isnan(got[2]).all() and (np.delete(got, 2, 0) == 0).all()


@pytest.mark.parametrize("C", [33, 1025, 9000])
def test_gradients_against_differences(C):
    """The kernel's own forward pass in float32 logits, along random directions:
    a central difference of step h is off by O(h^2) and the rounding 2 SUM / h."""
    z, g = make(C, 4, C, F32, std=1.0)
    tok = given(g, 4, C, 2)
    rng = np.random.default_rng(C)
    d_lp, d_ent = rng.normal(size=(4, 2)), rng.normal(size=4)
    grad = run_grad(z, tok, d_lp, None, d_ent)
    h = 0.02
    for _ in range(3):
        d = torch.tensor(rng.normal(size=(4, C)), dtype=F32).cuda()
        val = []
        for s in (h, -h):
            lp, _, ent, _, _ = score((z + s * d).contiguous(), tok, 0)
            val.append((lp * d_lp).sum() + (ent * d_ent).sum())
        got = (val[0] - val[1]) / (2 * h)
        size = np.abs(d_lp).sum() + np.abs(d_ent).sum()
        assert abs(got - (grad * d.cpu().numpy()).sum()) < size * (30 * h * h + 2 * SUM / h)


# ---------------------------------------------------------------------------
# distillation


def teacher(g, n, C, K, tail):
    """Lists of distinct tokens, some shorter, one empty, unused places anywhere."""
    ids = torch.stack([torch.randperm(C, generator=g)[:K] if C < 5000 else
                       torch.randint(0, C // 64, (K,), generator=g) * 64 + torch.arange(K) % 64
                       for _ in range(n)]).to(torch.int32)
    if ids.shape[1] < K:
        ids = torch.nn.functional.pad(ids, (0, K - ids.shape[1]), value=-1)
    sc = torch.randn((n, K), generator=g) * 2
    if tail:
        sc = torch.log_softmax(sc, 1) + torch.log(torch.linspace(0.3, 0.999, n))[:, None]
    if n > 2 and K > 1:
        ids[1, K // 2:] = -1
        ids[2, 0] = -1
    if n > 3:
        ids[3] = -1
    return ids, sc.contiguous()


def run_distill(z, ids, sc, tail, w=None, tau=1.0, loss=True, grad=True, in_place=False):
    from paper_2608_21343_amd import capi
    n, C = z.shape
    buf = torch.full((n, C + 3), 55.0, dtype=z.dtype, device="cuda")
    out = buf[:, :C]
    src = z
    if in_place:
        out.copy_(z)
        src = out
    o_loss = torch.full((n,), 77.0, device="cuda") if loss else None
    wt = None if w is None else torch.tensor(w, dtype=F32).cuda()
    capi.tb_distill(src, ids.cuda(), sc.cuda(), o_loss, out if grad else None, weight=wt,
                    temperature=tau, tail=tail)
    torch.cuda.synchronize()
    assert bool((buf[:, C:] == 55.0).all())
    return (o_loss.cpu().numpy() if loss else None, out.float().cpu().numpy() if grad else None)


def check_distill(z, ids, sc, tail, w=None, tau=1.0, in_place=False):
    loss, grad = run_distill(z, ids, sc, tail, w, tau, in_place=in_place)
    zh = host(z)
    scf = sc.numpy().astype(np.float64)
    want, dwant, p_rest = R.distill(zh, tau, ids.numpy(), scf, tail, w)
    n, C = z.shape
    wt = np.ones(n) if w is None else np.abs(w)
    with np.errstate(divide="ignore", invalid="ignore"):
        far = np.nan_to_num(np.abs(np.log(p_rest)), nan=0.0, posinf=0.0) if tail else np.zeros(n)
    # the teacher's own exponents are of the scores' size
    close(loss, want, wt * (SUM + 2e-5 + 1e-6 * (20 + far)), 1e-6)
    size = np.zeros((n, C))
    for i in range(n):
        used, q, _, mass, rest = R.teacher_row(ids.numpy()[i], scf[i], tau, tail, C)
        logp, lse = R.softmax_row(zh[i], tau)
        if not lse > NEG:
            continue
        p = np.exp(logp)
        extra = 0.0
        if tail and rest > 0 and p_rest[i] > 0:
            extra = (rest + 0.1) / p_rest[i]
        size[i] = p * (1 + extra)
        for (t, _), qk in zip(used, q):
            if 0 <= t < C:
                size[i, t] += qk
    size = size * (wt / tau)[:, None]
    close(grad, dwant, 1e-5 * size + 1e-37, 2.0 ** -7.99 if z.dtype == BF16 else REL)
    return loss, grad


@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("dtype, C", WIDTHS, ids=ids)
def test_distill_at_every_width(dtype, C, tail):
    n = 6 if C < 40000 else 2
    z, g = make(C, n, C, dtype, pad=1)
    K = min(8, C - 1)
    ids, sc = teacher(g, n, C, K, tail)
    loss, grad = check_distill(z, ids, sc, tail, tau=1.0 if tail else 2.0)
    only, _ = run_distill(z, ids, sc, tail, tau=1.0 if tail else 2.0, grad=False)
    np.testing.assert_array_equal(only, loss)
    _, alone = run_distill(z, ids, sc, tail, tau=1.0 if tail else 2.0, loss=False)
    np.testing.assert_array_equal(alone, grad)
    check_distill(z, ids, sc, tail, np.linspace(0, 2, n), 1.3, in_place=True)


@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("K", [1, 2, 5, 16, 33, 64])
@pytest.mark.parametrize("dtype, C", [(F32, 70), (BF16, 1025), (F32, 9000), (BF16, 140000)],
                         ids=ids)
def test_distill_lists(dtype, C, K, tail):
    z, g = make(K, 5, C, dtype)
    ids, sc = teacher(g, 5, C, K, tail)
    check_distill(z, ids, sc, tail)
    if K > 1:  # a token in two places
        ids[0, K - 1] = ids[0, 0]
        ids[4] = ids[4, 0]
        check_distill(z, ids, sc, tail)


@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("dtype, C", [(F32, 9), (F32, 1025), (BF16, 1025), (BF16, 8193),
                                      (F32, 20000), (F32, 70001)], ids=ids)
def test_distill_special_rows(dtype, C, tail):
    z = special_rows(C, dtype).cuda()
    n = z.shape[0]
    ids = torch.tensor([[C // 2, 0, C - 1]] * n, dtype=torch.int32)
    sc = torch.log(torch.tensor([[0.5, 0.2, 0.1]])).repeat(n, 1).contiguous()
    check_distill(z, ids, sc, tail)
    w = np.where(np.arange(n) % 2, 0.0, 1.5)
    loss, grad = check_distill(z, ids, sc, tail, w)
    assert (loss[1::2] == 0).all() and (grad[1::2] == 0).all()


def test_distill_whole_vocabulary_and_sure_teachers():
    """A list of every token (nothing is left outside), a teacher sure of one
    token, one with more mass than 1 by rounding, places of probability zero."""
    z, g = make(1, 4, 6, F32)
    ids = torch.arange(6, dtype=torch.int32).repeat(4, 1)
    sc = torch.log_softmax(torch.randn((4, 6), generator=g), 1)
    sc[1] = torch.tensor([0.0] + [NEG] * 5)
    sc[2] = torch.tensor([1e-6] + [NEG] * 5)
    check_distill(z, ids, sc, False)
    # exp of the scores sums to 1 but for rounding, and no token is left to take
    # a positive rest: rows whose list leaves tokens out are compared
    ids[:, 5] = -1
    sc[0] = torch.log_softmax(torch.randn(6, generator=g), 0)
    check_distill(z, ids, sc, True)


def test_distill_bad_tokens_and_scores():
    z, g = make(2, 5, 1025, F32)
    ids, sc = teacher(g, 5, 1025, 4, False)
    ids[3] = torch.tensor([1, 2, 3, 4])
    ids[0, 1], ids[1, 0] = 1025, -7
    sc[4, 2] = math.nan
    for tail in (False, True):
        loss, grad = run_distill(z, ids, sc, tail)
        for i in (0, 1, 4):
            assert np.isnan(loss[i]) and np.isnan(grad[i]).all()
        assert np.isfinite(loss[[2, 3]]).all() and np.isfinite(grad[[2, 3]]).all()


def test_alternatives_feed_distillation():
    """A teacher's alternatives, as they are written, are a list with its tail;
    a student equal to the teacher has loss 0 and no gradient."""
    from paper_2608_21343_amd import capi
    z, g = make(8, 9, 1025, F32)
    z[4] = NEG
    z[4, 7] = 1.0  # fewer tokens than places
    alt = torch.empty((9, 16), dtype=torch.int32, device="cuda")
    alt_lp = torch.empty((9, 16), device="cuda")
    capi.tb_token_logprobs(z, out_alt=alt, out_alt_logprob=alt_lp, temperature=1.5)
    loss = torch.empty(9, device="cuda")
    grad = torch.empty_like(z)
    capi.tb_distill(z, alt, alt_lp, loss, grad, temperature=1.5, tail=True)
    assert float(loss.abs().max()) < 3 * SUM and float(grad.abs().max()) < 3 * SUM


# ---------------------------------------------------------------------------
# offsets, streams, graphs


def test_rows_beyond_32_bits():
    """Rows whose offsets pass 2^31 and 2^32 elements."""
    from paper_2608_21343_amd import capi
    C, stride = 1025, 1 << 26
    n = 70
    buf = torch.empty(stride * (n - 1) + C, dtype=BF16, device="cuda")
    z = buf.as_strided((n, C), (stride, 1))
    small, g = make(9, n, C, BF16)
    z.copy_(small)
    tok = given(g, n, C, 2)
    a, b = score(z, tok, 8), score(small, tok, 8)
    for x, y in zip(a, b):
        np.testing.assert_array_equal(x, y)
    d = torch.ones((n, 2), device="cuda")
    want = torch.empty_like(small)
    capi.tb_token_logprobs_grad(small, tok.cuda(), d, want)
    capi.tb_token_logprobs_grad(z, tok.cuda(), d, z)
    assert bool((z == want).all())


def test_many_rows():
    """More rows than a launch of one workgroup per row may have work-items for
    (two columns: the smallest row), against the same rows in a short call."""
    from paper_2608_21343_amd import capi
    n = (1 << 26) + 5
    z = torch.randn(8, 2).cuda()
    big = z.repeat((n + 7) // 8, 1)[:n].contiguous()
    lse = torch.empty(n, device="cuda")
    few = torch.empty(8, device="cuda")
    capi.tb_token_logprobs(big, out_lse=lse)
    capi.tb_token_logprobs(z, out_lse=few)
    assert bool((lse[:n // 8 * 8].view(-1, 8) == few).all()) and bool((lse[-5:] == few[:5]).all())


def test_results_are_the_same_each_time_and_on_other_streams():
    from paper_2608_21343_amd import capi
    for dtype, C in ((F32, 1025), (BF16, 9000), (F32, 100001)):
        z, g = make(10, 6, C, dtype)
        tok = given(g, 6, C, 2)
        ids, sc = teacher(g, 6, C, 8, True)
        first = score(z, tok, 16)
        dist = run_distill(z, ids, sc, True)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        lp = torch.empty((6, 2), device="cuda")
        loss, grad = torch.empty(6, device="cuda"), torch.empty_like(z)
        args = (tok.cuda(), ids.cuda(), sc.cuda())
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            capi.tb_token_logprobs(z, args[0], lp)
            capi.tb_distill(z, args[1], args[2], loss, grad, tail=True)
        st.synchronize()
        np.testing.assert_array_equal(lp.cpu().numpy(), first[0])
        np.testing.assert_array_equal(loss.cpu().numpy(), dist[0])
        np.testing.assert_array_equal(grad.float().cpu().numpy(), dist[1])
        for x, y in zip(score(z, tok, 16), first):
            np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("dtype, C", [(F32, 1025), (F32, 100001)], ids=ids)
def test_captured_in_a_graph(dtype, C):
    from paper_2608_21343_amd import capi
    z, g = make(11, 5, C, dtype)
    tok = given(g, 5, C, 1).cuda()
    alt = torch.empty((5, 8), dtype=torch.int32, device="cuda")
    alt_lp = torch.empty((5, 8), device="cuda")
    lp, loss = torch.empty((5, 1), device="cuda"), torch.empty(5, device="cuda")
    grad = torch.empty_like(z)
    need = capi.tb_rows_workspace_bytes(z, 8)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None

    def step():
        capi.tb_token_logprobs(z, tok, lp, None, None, alt, alt_lp, workspace=ws)
        capi.tb_distill(z, alt, alt_lp, loss, grad, temperature=2.0, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        z.copy_(make(20 + k, 5, C, dtype)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (lp, alt, alt_lp, loss, grad)]
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, (lp, alt, alt_lp, loss, grad)):
            assert bool((x == y).all())

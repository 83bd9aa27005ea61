"""The float64 forms of the row operators against torch's float64 autograd,
closed forms and differences; and the refusals of the C entry points, which come
before anything is launched."""

import math

import numpy as np
import pytest
import torch

from tests import rows_reference as R


def _case(seed, n=5, V1=23, K=4):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(n, V1)) * 2
    ids = np.stack([rng.permutation(V1)[:K] for _ in range(n)]).astype(np.int32)
    return rng, z, ids


@pytest.mark.parametrize("tau", [1.0, 0.5, 3.0])
def test_scores_are_log_softmax(tau):
    rng, z, ids = _case(1)
    lp, lse, ent, alt, alt_lp = R.scores(z, tau, ids, 6)
    u = torch.tensor(z / tau)
    ref = torch.log_softmax(u, 1)
    np.testing.assert_allclose(lp, torch.gather(ref, 1, torch.tensor(ids).long()), rtol=1e-13)
    np.testing.assert_allclose(lse, torch.logsumexp(u, 1), rtol=1e-13)
    np.testing.assert_allclose(ent, -(ref.exp() * ref).sum(1), rtol=1e-13)
    np.testing.assert_array_equal(alt, torch.topk(u, 6, dim=1).indices)
    np.testing.assert_allclose(alt_lp, torch.topk(ref, 6, dim=1).values, rtol=1e-13)


def test_scores_of_uniform_and_masked_rows():
    z = np.array([[0.0] * 8, [R.NEG] * 8, [R.NEG] * 6 + [2.0, 2.0]])
    lp, lse, ent, alt, alt_lp = R.scores(z, 1.0, np.array([[0, -1]] * 3, np.int32), 3)
    np.testing.assert_allclose(lp[0], [-math.log(8), 0.0])
    np.testing.assert_allclose(ent, [math.log(8), 0.0, math.log(2)])
    assert alt.tolist() == [[0, 1, 2], [-1, -1, -1], [6, 7, -1]]
    assert lse[1] == R.NEG and lp[1].tolist() == [R.NEG, 0.0] and alt_lp[2][2] == R.NEG


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_gradients_are_autograd(tau):
    rng, z, ids = _case(2)
    ids[:, 1] = ids[:, 0]  # a token listed twice
    g, gl, gh = rng.normal(size=ids.shape), rng.normal(size=5), rng.normal(size=5)
    x = torch.tensor(z, requires_grad=True)
    logp = torch.log_softmax(x / tau, 1)
    ent = -(logp.exp() * logp).sum(1)
    val = (torch.gather(logp, 1, torch.tensor(ids).long()) * torch.tensor(g)).sum()
    (val + (torch.logsumexp(x / tau, 1) * torch.tensor(gl)).sum()
     + (ent * torch.tensor(gh)).sum()).backward()
    np.testing.assert_allclose(R.score_grad(z, tau, ids, g, gl, gh), x.grad, atol=1e-13)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distillation_is_autograd_and_differences(tail, tau):
    rng, z, ids = _case(3)
    ids[1, 2:] = -1
    ids[2] = -1
    score = rng.normal(size=ids.shape)
    if tail:
        score = np.log(0.8 * np.exp(score) / np.exp(score).sum(1, keepdims=True))
    w = np.array([1.0, 0.5, 2.0, 0.0, 3.0])
    loss, grad, _ = R.distill(z, tau, ids, score, tail, w)
    x = torch.tensor(z, requires_grad=True)
    logp = torch.log_softmax(x / tau, 1)
    total = 0.0
    for i in range(5):
        at = [j for j in range(ids.shape[1]) if ids[i, j] >= 0]
        s = torch.tensor(score[i, at])
        logq = s if tail else torch.log_softmax(s / tau, 0)
        k = (logq.exp() * (logq - logp[i, ids[i, at]])).sum() if at else 0.0
        if tail:
            out = [v for v in range(z.shape[1]) if v not in set(ids[i, at].tolist())]
            rest = 1 - logq.exp().sum()
            k = k + rest * (torch.log(rest) - torch.log(logp[i, out].exp().sum()))
        np.testing.assert_allclose(loss[i], w[i] * float(k.detach() if at else k), atol=1e-13)
        total = total + w[i] * k
    total.backward()
    np.testing.assert_allclose(grad, x.grad, atol=1e-13)
    d = rng.normal(size=z.shape)
    h = 1e-6
    up = R.distill(z + h * d, tau, ids, score, tail, w)[0].sum()
    down = R.distill(z - h * d, tau, ids, score, tail, w)[0].sum()
    assert abs((up - down) / (2 * h) - (grad * d).sum()) < 1e-7


# ---------------------------------------------------------------------------
# refusals: every one of these returns before a launch, so that addresses of
# no device memory serve

BUF = 1 << 20  # distances between the made-up buffers


def _addr(i):
    return 0x10000000 + i * BUF


def _logprobs(**kw):
    a = dict(logits=_addr(0), dtype=0, n=2, v1=9, stride=9, tau=1.0, tok=_addr(1), J=1,
             lp=_addr(2), lse=_addr(3), ent=_addr(4), M=2, alt=_addr(5), alt_lp=_addr(6), ws=None,
             wsb=0)
    a.update(kw)
    from paper_2608_21343_amd import capi
    r = capi.LIB.tb_token_logprobs(a["logits"], a["dtype"], a["n"], a["v1"], a["stride"], a["tau"],
                                   a["tok"], a["J"], a["lp"], a["lse"], a["ent"], a["M"], a["alt"],
                                   a["alt_lp"], a["ws"], a["wsb"], None)
    return r, capi.LIB.tb_last_error().decode()


def _grad(**kw):
    a = dict(logits=_addr(0), dtype=0, n=2, v1=9, stride=9, tau=1.0, tok=_addr(1), J=1,
             d_lp=_addr(2), d_lse=_addr(3), d_ent=_addr(4), grad=_addr(5), gs=9, ws=None, wsb=0)
    a.update(kw)
    from paper_2608_21343_amd import capi
    r = capi.LIB.tb_token_logprobs_grad(a["logits"], a["dtype"], a["n"], a["v1"], a["stride"],
                                        a["tau"], a["tok"], a["J"], a["d_lp"], a["d_lse"],
                                        a["d_ent"], a["grad"], a["gs"], a["ws"], a["wsb"], None)
    return r, capi.LIB.tb_last_error().decode()


def _distill(**kw):
    a = dict(logits=_addr(0), dtype=0, n=2, v1=9, stride=9, tau=1.0, tok=_addr(1), sc=_addr(2),
             K=2, tail=0, w=_addr(3), loss=_addr(4), grad=_addr(5), gs=9, ws=None, wsb=0)
    a.update(kw)
    from paper_2608_21343_amd import capi
    r = capi.LIB.tb_distill(a["logits"], a["dtype"], a["n"], a["v1"], a["stride"], a["tau"],
                            a["tok"], a["sc"], a["K"], a["tail"], a["w"], a["loss"], a["grad"],
                            a["gs"], a["ws"], a["wsb"], None)
    return r, capi.LIB.tb_last_error().decode()


SHARED = [
    (dict(n=-1), "n_rows"), (dict(n=1 << 41), "n_rows"), (dict(dtype=2), "dtype"),
    (dict(v1=1), "v_plus_blank"), (dict(v1=(1 << 20) + 1, stride=1 << 21), "v_plus_blank"),
    (dict(stride=8), "row_stride"), (dict(n=1 << 40, stride=1 << 30), "row_stride"),
    (dict(logits=None), "logits"), (dict(logits=_addr(0) + 2), "logits"),
    (dict(logits=_addr(0) + 1, dtype=1), "logits"), (dict(tau=0.0), "temperature"),
    (dict(tau=-1.0), "temperature"), (dict(tau=math.nan), "temperature"),
    (dict(tau=math.inf), "temperature"), (dict(tok=_addr(1) + 2), "aligned"),
    (dict(tok=None), "NULL"),
]


@pytest.mark.parametrize("call", [_logprobs, _grad, _distill])
@pytest.mark.parametrize("change, word", SHARED)
def test_shared_refusals(call, change, word):
    r, msg = call(**change)
    assert r == -1 and word in msg, (r, msg)


@pytest.mark.parametrize("call, change, word", [
    (_logprobs, dict(J=65), "n_tok"), (_logprobs, dict(J=-1), "n_tok"),
    (_logprobs, dict(M=65), "n_alt"), (_logprobs, dict(lp=None), "out_logprob"),
    (_logprobs, dict(alt=None), "out_alt"), (_logprobs, dict(alt_lp=None), "out_alt_logprob"),
    (_logprobs, dict(lse=_addr(3) + 1), "out_lse"), (_logprobs, dict(lse=_addr(4)), "overlaps"),
    (_logprobs, dict(lp=_addr(0) + 8), "overlaps"), (_logprobs, dict(alt=_addr(1)), "overlaps"),
    (_grad, dict(J=65), "n_tok"), (_grad, dict(d_lp=None), "d_logprob"),
    (_grad, dict(grad=None), "grad"), (_grad, dict(grad=_addr(5) + 2), "grad"),
    (_grad, dict(gs=8), "grad_stride"), (_grad, dict(grad=_addr(0) + 4), "overlaps"),
    (_grad, dict(grad=_addr(0), gs=10), "overlaps"), (_grad, dict(grad=_addr(2)), "overlaps"),
    (_grad, dict(d_ent=_addr(4) + 2), "d_entropy"),
    (_distill, dict(K=0), "n_teacher"), (_distill, dict(K=65), "n_teacher"),
    (_distill, dict(tail=2), "tail"), (_distill, dict(sc=None), "teacher_score"),
    (_distill, dict(w=_addr(3) + 2), "weight"), (_distill, dict(loss=None, grad=None), "both"),
    (_distill, dict(loss=_addr(3)), "overlaps"), (_distill, dict(grad=_addr(0) + 36), "overlaps"),
    (_distill, dict(grad=_addr(0), loss=_addr(0) + 4), "overlaps"),
])
def test_refusals(call, change, word):
    r, msg = call(**change)
    assert r == -1 and word in msg, (r, msg)


@pytest.mark.parametrize("call", [_logprobs, _grad, _distill])
def test_rows_in_segments_need_a_workspace(call):
    from paper_2608_21343_amd import capi
    v1 = 1 << 20
    M = 2 if call is _logprobs else 0
    need = capi.LIB.tb_rows_workspace_bytes(0, 2, v1, M)
    assert need > 0
    far = {"logits": 1 << 40, "v1": v1, "stride": v1}
    if call is not _logprobs:
        far.update(grad=1 << 41, gs=v1)
    for kw in (dict(), dict(ws=1 << 42, wsb=need - 1)):
        r, msg = call(**far, **kw)
        assert r == -2 and "workspace" in msg
    r, msg = call(**far, ws=(1 << 42) + 4, wsb=need)
    assert r == -1 and "aligned" in msg
    r, msg = call(**far, ws=1 << 40, wsb=need)
    assert r == -1 and "overlaps" in msg


@pytest.mark.parametrize("call", [_logprobs, _grad, _distill])
def test_no_rows_touch_nothing(call):
    r, _ = call(n=0, logits=None, tok=None)
    assert r == 0


def test_workspace_bytes():
    from paper_2608_21343_amd import capi
    f = capi.LIB.tb_rows_workspace_bytes
    assert f(0, 1000, 1025, 64) == 0 and f(0, 0, 1 << 20, 64) == 0
    assert f(0, 10, 1 << 20, 8) >= f(0, 10, 1 << 20, 0) > 0
    for bad in ((2, 1, 9, 0), (0, -1, 9, 0), (0, 1, 1, 0), (0, 1, (1 << 20) + 1, 0), (0, 1, 9, 65),
                (0, 1, 9, -1)):
        assert f(*bad) == -1


def test_binding_refuses_host_tensors_and_shapes():
    from paper_2608_21343_amd import capi
    z = torch.zeros(3, 9)
    with pytest.raises(ValueError, match="device"):
        capi.tb_token_logprobs(z)
    with pytest.raises(ValueError, match="contiguous"):
        capi.tb_token_logprobs(z[:, ::2])
    with pytest.raises(ValueError, match="evenly"):
        capi.tb_token_logprobs(torch.zeros(3, 4, 9)[:, :3])
    with pytest.raises(ValueError, match="overlap"):
        capi.tb_token_logprobs(torch.zeros(9).expand(3, 9))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        capi.tb_token_logprobs(z.double())

"""Plain float64 forms of the row operators, a row at a time, from their
definitions (numpy; shares no code with the library)."""

import math

import numpy as np

NEG = -math.inf


def softmax_row(z, tau):
    """(log probabilities, lse) of one row; an empty row has none; a row with a
    NaN or +inf has NaN."""
    u = np.asarray(z, np.float64) / tau
    if np.isnan(u).any() or (u == math.inf).any():
        return np.full(u.shape, np.nan), math.nan
    m = u.max()
    if m == NEG:
        return np.full(u.shape, NEG), NEG
    log_s = math.log(np.exp(u - m).sum())
    return (u - m) - log_s, m + log_s  # u - lse would lose log_s beside a large m


def entropy_row(logp):
    p = np.exp(logp)
    return float(np.sum(np.where(p > 0, -p * np.where(p > 0, logp, 0.0), p * 0.0)))


def top_row(z, n):
    """Ids of the n largest, ties to the lowest id, only above -inf; -1 beyond."""
    z = np.asarray(z, np.float64)
    ok = np.flatnonzero(z > NEG)  # a NaN is not
    order = ok[np.lexsort((ok, -z[ok]))][:n]
    return np.concatenate([order, np.full(n - len(order), -1)]).astype(np.int32)


def scores(z, tau, tokens, n_alt):
    """(logprob, lse, entropy, alt, alt_logprob) of rows z [n, C]."""
    n, C = z.shape
    lp = np.zeros(tokens.shape)
    lse, ent = np.zeros(n), np.zeros(n)
    alt = np.zeros((n, n_alt), np.int32)
    alt_lp = np.zeros((n, n_alt))
    for i in range(n):
        logp, lse[i] = softmax_row(z[i], tau)
        ent[i] = entropy_row(logp)
        for j, t in enumerate(tokens[i]):
            lp[i, j] = 0.0 if t == -1 else logp[t] if 0 <= t < C else math.nan
        alt[i] = top_row(z[i], n_alt)
        alt_lp[i] = [logp[t] if t >= 0 else NEG for t in alt[i]]
    return lp, lse, ent, alt, alt_lp


def score_grad(z, tau, tokens, d_lp, d_lse, d_ent):
    """Gradient with respect to z of sum(d_lp * logprob) + d_lse lse + d_ent entropy."""
    n, C = z.shape
    out = np.zeros((n, C))
    for i in range(n):
        used = [(t, g) for t, g in zip(tokens[i], d_lp[i]) if t != -1]
        bad = any(not 0 <= t < C for t, _ in used)
        gl = 0.0 if d_lse is None else float(d_lse[i])
        gh = 0.0 if d_ent is None else float(d_ent[i])
        if not bad and gl == 0 and gh == 0 and all(g == 0 for _, g in used):
            continue
        logp, lse = softmax_row(z[i], tau)
        if bad:
            out[i] = math.nan
            continue
        if lse == NEG:
            continue
        p = np.exp(logp)
        d = p * (gl - sum(float(g) for _, g in used))
        if gh:
            d = d - gh * p * np.where(p > 0, np.where(p > 0, logp, 0.0) + entropy_row(logp), p * 0)
        for t, g in used:
            d[t] += float(g)
        out[i] = d / tau
    return out


def teacher_row(ids, score, tau, tail, C):
    """(used places, q, log q, mass of the list, rest)."""
    used = [(int(t), float(s)) for t, s in zip(ids, score) if t != -1]
    s = np.array([x for _, x in used])
    if tail:
        q = np.exp(s)
        return used, q, s, q.sum(), max(0.0, 1.0 - q.sum())
    if not len(s) or s.max() == NEG:
        return used, np.zeros(len(s)), s, 0.0, 0.0
    logq = s / tau - s.max() / tau
    logq = logq - math.log(np.exp(logq).sum())
    return used, np.exp(logq), logq, 1.0, 0.0


def distill(z, tau, ids, score, tail, weight):
    """(loss [n], gradient [n, C], p_rest [n])."""
    n, C = z.shape
    loss, grad, p_rest = np.zeros(n), np.zeros((n, C)), np.ones(n)
    for i in range(n):
        w = 1.0 if weight is None else float(weight[i])
        used, q, logq, mass, rest = teacher_row(ids[i], score[i], tau, tail, C)
        bad = any(not 0 <= t < C for t, _ in used)
        if w == 0 or (mass + rest == 0 and not bad):
            continue
        if bad:
            loss[i] = math.nan
            grad[i] = math.nan
            continue
        logp, lse = softmax_row(z[i], tau)
        p = np.exp(logp)
        listed = np.zeros(C, bool)
        listed[[t for t, _ in used]] = True
        total = sum(qk * (lq - logp[t]) for (t, _), qk, lq in zip(used, q, logq) if qk > 0)
        p_rest[i] = p[~listed].sum()
        d = (mass + rest) * p
        if rest > 0:
            total += rest * (math.log(rest) - (math.log(p_rest[i]) if p_rest[i] > 0 else
                                               p_rest[i] * 0 + NEG))
            if p_rest[i] > 0 or math.isnan(p_rest[i]):
                d[~listed] -= rest * p[~listed] / p_rest[i]
        for (t, _), qk in zip(used, q):
            d[t] -= qk
        loss[i] = w * total
        grad[i] = 0.0 if lse == NEG else w * d / tau
    return loss, grad, p_rest

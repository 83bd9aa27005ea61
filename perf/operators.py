"""The row operators of this library as timed cases: log probabilities of given
tokens with entropy and top alternatives, their gradient, and the distillation
loss from a teacher's top logits with its gradient.

A case is a plain dict:

* ``op``: "score" (log probabilities, log-sum-exp, entropy, alternatives),
  "score_grad" (the logits' gradient from the outputs' gradients),
  "distill" (loss per row) or "distill_grad" (loss per row and gradient);
* ``rows`` rows of ``V`` tokens and the blank, of type ``dtype``, padded by
  ``pad`` values, taken at ``temperature``;
* ``tokens`` given tokens a row (-1: none), ``alts`` alternatives a row,
  ``entropy``: whether the entropy has a gradient;
* ``teacher`` teacher tokens a row, ``tail``: whether the teacher's scores are
  log probabilities whose missing mass counts, ``weighted``: whether rows have
  weights (some of them 0, as padding frames have);
* ``masked``: rows in which most tokens are masked, with -inf or the type's
  lowest value, and some in which all are.

``run`` makes one pass: the plain form in 32 bits from elementary operations,
or with ``own`` the library's calls.
"""

from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

_BASE = dict(op="score", rows=1, V=1024, dtype="f32", pad=0, temperature=1.0, tokens=0, alts=0,
             entropy=False, teacher=0, tail=False, weighted=False, masked=False)


def listed():
    return [
        # confidences of one step of 128 live streams: latency of a single call
        dict(_BASE, name="score_step", rows=128, tokens=1, alts=4),
        # the same over a chunk of 16 steps, label against blank
        dict(_BASE, name="score_chunk", rows=2048, tokens=2, alts=8),
        # a batch of long recordings, scored offline
        dict(_BASE, name="score_long", rows=131072, tokens=1, alts=8),
        # a teacher's alternatives over a large vocabulary, to be distilled from
        dict(_BASE, name="score_wide", rows=65536, V=8192, dtype="bf16", tokens=1, alts=32),
        # odd sizes, padded rows, masked tokens and empty rows, softened
        dict(_BASE, name="score_odd", rows=7511, V=611, dtype="bf16", pad=5, temperature=1.7,
             tokens=3, alts=5, masked=True),
        # single tokens of a few streams over a text vocabulary
        dict(_BASE, name="score_vocab", rows=8, V=131072, tokens=1, alts=20),
        # training on a batch of utterances: label and blank, with an entropy term
        dict(_BASE, name="grad_batch", op="score_grad", rows=16000, tokens=2, entropy=True),
        # the log-likelihood's gradient over a large vocabulary
        dict(_BASE, name="grad_wide", op="score_grad", rows=16384, V=8192, dtype="bf16",
             tokens=1),
        # a training step against eight softened teacher logits a frame
        dict(_BASE, name="distill_batch", op="distill_grad", rows=16384, teacher=8,
             temperature=2.0),
        # odd sizes, padded rows, masked tokens, rows of weight 0, the teacher's tail
        dict(_BASE, name="distill_odd", op="distill_grad", rows=7511, V=611, dtype="bf16", pad=5,
             teacher=5, tail=True, weighted=True, masked=True),
        # the loss alone over a validation set
        dict(_BASE, name="distill_check", op="distill", rows=32768, dtype="bf16", teacher=16,
             tail=True),
        # a text vocabulary with long teacher lists
        dict(_BASE, name="distill_vocab", op="distill_grad", rows=2048, V=131072, dtype="bf16",
             teacher=64, tail=True, weighted=True),
    ]


#: The logits of the largest listed case of each operator, in values.
MOST_VALUES = {"score": 65536 * 8193, "score_grad": 16384 * 8193, "distill": 2048 * 131073,
               "distill_grad": 2048 * 131073}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_BASE)
    c["op"] = rng.choice(["score", "score", "score_grad", "distill", "distill_grad",
                          "distill_grad"])
    c["dtype"] = rng.choice(["f32", "bf16"])
    c["V"] = _log_int(rng, 200, 131072)
    c["rows"] = _log_int(rng, 1, 131072)
    c["rows"] = max(1, min(c["rows"], MOST_VALUES[c["op"]] // (4 * (c["V"] + 1))))
    c["pad"] = rng.choice([0, 0, 0, 3, 7, 64])
    c["temperature"] = rng.choice([1.0, 1.0, 0.7, 2.0, 4.0])
    c["masked"] = rng.random() < 0.25
    if c["op"] in ("score", "score_grad"):
        c["tokens"] = rng.choice([1, 1, 2, 2, 3, 5, 16, 64])
    if c["op"] == "score":
        c["alts"] = rng.choice([0, 1, 4, 5, 8, 8, 10, 16, 20, 32, 64])
    if c["op"] == "score_grad":
        c["entropy"] = rng.random() < 0.5
    if c["op"] in ("distill", "distill_grad"):
        c["teacher"] = rng.choice([1, 4, 5, 8, 8, 16, 20, 32, 64])
        c["tail"] = rng.random() < 0.5
        c["weighted"] = rng.random() < 0.5
    return c


# ---------------------------------------------------------------------------
# inputs


def _rows(c, g):
    """Logits as a joint or a language model gives them: a spread of unlikely
    tokens, one that most rows clearly prefer, and a blank (the last id) ahead
    of the average token. Also that preferred token of every row."""
    n, C = c["rows"], c["V"] + 1
    buf = torch.empty((n, C + c["pad"]), dtype=DTYPES[c["dtype"]], device="cuda")
    z = torch.randn((n, C), generator=g, device="cuda")
    z *= 1.5
    z[:, C - 1] += 2.0
    best = torch.randint(0, C, (n, 1), generator=g, device="cuda")
    z.scatter_add_(1, best, 2.0 + 8.0 * torch.rand((n, 1), generator=g, device="cuda"))
    buf.fill_(1e4)
    buf[:, :C] = z
    return buf[:, :C], best


def _mask(z, visible, g):
    """A sixth of the rows show few tokens, the others at -inf, another sixth
    with the others at the type's lowest value, and some show none at all."""
    n, C = z.shape
    kind = torch.randint(0, 6, (n, 1), generator=g, device="cuda")
    keep = torch.rand((n, C), generator=g, device="cuda") < 0.03
    keep.scatter_(1, visible.clamp(min=0).long(), True)
    none = (kind == 2) & (torch.rand((n, 1), generator=g, device="cuda") < 0.2)
    z.masked_fill_(~keep & (kind == 0) | none, -math.inf)
    z.masked_fill_(~keep & (kind == 1), torch.finfo(z.dtype).min)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    n, C = c["rows"], c["V"] + 1
    z, best = _rows(c, g)
    s = dict(c, z=z)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    J, M, K = c["tokens"], c["alts"], c["teacher"]
    if J:
        # the preferred token or the blank first, then any; some rows have fewer
        tok = torch.randint(0, C, (n, J), generator=g, device="cuda")
        tok[:, :1] = torch.where(uniform(n, 1) < 0.7, best, C - 1)
        tok[:, -1:] = torch.where(uniform(n, 1) < 0.1, -1, tok[:, -1:])
        s["tok"] = tok.to(torch.int32)
    if c["op"] == "score_grad":
        s["d_logprob"] = -uniform(n, J) / n
        s["d_entropy"] = 0.1 * normal(n) / n if c["entropy"] else None
    if K:
        # a teacher that mostly agrees: its K best of some hundred tokens around
        # the preferred one
        share = min(C, max(4 * K, 512))
        first = best + torch.randint(0, share, (n, 1), generator=g, device="cuda") + (C - share)
        ids = (first + 1 + torch.arange(share, device="cuda")) % C
        t = normal(n, share) * 2.0 + torch.where(ids == best, 6.0, 0.0)
        t, at = torch.topk(t, K, dim=1)
        ids = torch.gather(ids, 1, at)
        if c["tail"]:
            t = torch.log_softmax(t, dim=1) + torch.log(0.6 + 0.399 * uniform(n, 1))
        # a tenth of the rows have a shorter list, a few none
        short = torch.where(uniform(n, 1) < 0.1, (uniform(n, 1) * K).floor(), float(K))
        ids = torch.where(torch.arange(K, device="cuda") < short, ids, -1)
        s["teacher_tok"] = ids.to(torch.int32)
        s["teacher_score"] = t.contiguous()
        s["weight"] = None
        if c["weighted"]:
            s["weight"] = torch.where(uniform(n) < 0.2, 0.0, uniform(n) / n)
    if c["masked"]:
        _mask(z, s["tok"] if J else s["teacher_tok"], g)
    # the buffers that a program keeps for the results
    f32 = dict(dtype=torch.float32, device="cuda")
    if c["op"] == "score":
        s["out"] = (torch.empty((n, J), **f32), torch.empty(n, **f32), torch.empty(n, **f32),
                    torch.empty((n, M), dtype=torch.int32, device="cuda") if M else None,
                    torch.empty((n, M), **f32) if M else None)
    if K:
        s["loss"] = torch.empty(n, **f32)
    if c["op"] in ("score_grad", "distill_grad"):
        s["grad"] = torch.empty((n, C), dtype=z.dtype, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2608_21343_amd import capi

    t = s["temperature"]
    if s["op"] == "score":
        lp, lse, ent, alt, alt_lp = s["out"]
        capi.tb_token_logprobs(s["z"], s["tok"], lp, lse, ent, alt, alt_lp, temperature=t)
        return {"logprob": lp, "lse": lse, "entropy": ent, "alt": alt, "alt_logprob": alt_lp}
    if s["op"] == "score_grad":
        capi.tb_token_logprobs_grad(s["z"], s["tok"], s["d_logprob"], s["grad"],
                                    d_entropy=s["d_entropy"], temperature=t)
        return {"grad": s["grad"]}
    capi.tb_distill(s["z"], s["teacher_tok"], s["teacher_score"], s["loss"], s.get("grad"),
                    weight=s["weight"], temperature=t, tail=s["tail"])
    if s["op"] == "distill":
        return {"loss": s["loss"]}
    return {"loss": s["loss"], "grad": s["grad"]}


def _softmax(z, temperature):
    """(z as float32, u - max u, their exponentials, sum, max u); rows without
    a value above -inf have sum 1 and no probabilities."""
    z = z.float()
    u = z / temperature if temperature != 1.0 else z
    m = u.amax(1, keepdim=True)
    x = u - torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    return z, x, e, torch.where(m == -math.inf, 1.0, total), m


def _at(x, ids):
    return torch.gather(x, 1, ids.clamp(min=0).long())


def _entropy(x, e, total):
    return total.log() - torch.where(e > 0, e * x, 0.0).sum(1, keepdim=True) / total


def _top(z, M):
    """Ids and values of the M largest by (value, lowest id): unique whole keys."""
    C = z.shape[1]
    bits = (z + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    key = key * (1 << 32) + torch.arange(0xffffffff, 0xffffffff - C, -1, device=z.device)
    key = torch.topk(key, min(M, C), dim=1).values
    ids = 0xffffffff - (key & 0xffffffff)
    if M > C:
        ids = torch.cat([ids, ids.new_full((ids.shape[0], M - C), -1)], 1)
    val = torch.where(ids >= 0, _at(z, ids), -math.inf)
    return torch.where(val > -math.inf, ids, -1).to(torch.int32), val


def _scatter_add(x, ids, add):
    return x.scatter_add_(1, ids.clamp(min=0).long(), torch.where(ids >= 0, add, 0.0))


def _run_plain(s):
    t = s["temperature"]
    dtype = s["z"].dtype
    z, x, e, total, m = _softmax(s["z"], t)
    log_total = total.log()
    if s["op"] == "score":
        lse = (log_total + m)[:, 0]
        lp = torch.where(s["tok"] >= 0, _at(x, s["tok"]) - log_total, 0.0)
        out = {"logprob": lp, "lse": lse, "entropy": _entropy(x, e, total)[:, 0]}
        if not s["alts"]:
            return dict(out, alt=None, alt_logprob=None)
        alt, val = _top(z, s["alts"])
        top = (val / t if t != 1.0 else val) - torch.where(m == -math.inf, 0.0, m)
        return dict(out, alt=alt, alt_logprob=top - log_total)
    p = e / total
    if s["op"] == "score_grad":
        used = torch.where(s["tok"] >= 0, s["d_logprob"], 0.0)
        d = -p * used.sum(1, keepdim=True)
        if s["d_entropy"] is not None:
            slope = torch.where(e > 0, x - log_total + _entropy(x, e, total), 0.0)
            d -= p * slope * s["d_entropy"][:, None]
        d = _scatter_add(d, s["tok"], torch.where(m > -math.inf, used, 0.0))
        return {"grad": (d / t).to(dtype)}
    ids, sc = s["teacher_tok"], s["teacher_score"].float()
    sc = torch.where(ids >= 0, sc, -math.inf)
    logp = torch.where(ids >= 0, _at(x, ids) - log_total, 0.0)
    if s["tail"]:
        q, logq = sc.exp(), sc
        rest = (1.0 - q.sum(1, keepdim=True)).clamp(min=0.0)
        seen = _scatter_add(torch.zeros_like(e), ids, 1.0) > 0
        p_rest = torch.where(seen, 0.0, e).sum(1, keepdim=True) / total
        loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1, keepdim=True)
        loss += torch.where(rest > 0, rest * (rest.log() - p_rest.log()), 0.0)
        ratio = torch.where(rest > 0, rest / p_rest, 0.0)
        mass = q.sum(1, keepdim=True) + rest
        d = torch.where(seen, mass * p, torch.where(e > 0, p * (mass - ratio), 0.0))
    else:
        sc = sc / t
        top = sc.amax(1, keepdim=True)
        w = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
        q_total = w.sum(1, keepdim=True)
        mass = (q_total > 0).float()
        q = w / torch.where(q_total > 0, q_total, 1.0)
        logq = sc - torch.where(top == -math.inf, 0.0, top) - q_total.log()
        loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1, keepdim=True)
        d = mass * p
    weight = s["weight"]
    if weight is not None:
        loss = torch.where(weight[:, None] != 0, loss * weight[:, None], 0.0)
    if s["op"] == "distill":
        return {"loss": loss[:, 0]}
    d = _scatter_add(d, ids, torch.where(m > -math.inf, -q, 0.0))
    if weight is not None:
        d = torch.where(weight[:, None] != 0, d * weight[:, None], 0.0)
    return {"loss": loss[:, 0], "grad": (d / t).to(dtype)}


# ---------------------------------------------------------------------------
# what a pass cannot do without


def work(c):
    n, C, size = c["rows"], c["V"] + 1, 4 if c["dtype"] == "f32" else 2
    J, M, K = c["tokens"], c["alts"], c["teacher"]
    values = n * C
    moved, ops = values * size, 5 * values  # maximum, difference, exponential, sum
    if c["op"] == "score":
        moved += n * (8 * J + 8 + 8 * M)
        ops += 3 * values
    if c["op"] == "score_grad":
        moved += values * size + n * (8 * J + (4 if c["entropy"] else 0))
        ops += (6 if c["entropy"] else 2) * values
    if K:
        moved += n * (8 * K + 4 + (4 if c["weighted"] else 0))
    if c["op"] == "distill_grad":
        moved += values * size
        ops += 2 * values
    return {"bytes": moved, "flops": ops}


# ---------------------------------------------------------------------------
# the definitions in 64 bits


def exact(c, seed):
    """Row by row from the definitions in float64: z / temperature, its
    log-softmax, and what each operator takes of it."""
    s = prepare(c, seed)
    tau, NEG = c["temperature"], -math.inf
    outs = []
    step = max(1, (1 << 26) // (c["V"] + 1))
    for a in range(0, c["rows"], step):
        rows = slice(a, a + step)
        u = s["z"][rows].double() / tau
        lse = torch.logsumexp(u, dim=1)
        empty = lse == NEG
        logp = torch.where(empty[:, None], NEG, u - torch.where(empty, 0.0, lse)[:, None])
        p = torch.exp(logp)
        plogp = torch.special.entr(p)  # -p log p, 0 at p = 0
        if c["op"] in ("score", "score_grad"):
            tok = s["tok"][rows].long()
            have = tok >= 0
        if c["op"] == "score":
            lp = torch.where(have, torch.gather(logp, 1, torch.where(have, tok, 0)), 0.0)
            M = min(c["alts"], c["V"] + 1)
            top = torch.topk(logp, M, dim=1).values
            top = torch.nn.functional.pad(top, (0, c["alts"] - M), value=NEG)
            outs.append({"logprob": lp, "lse": lse, "entropy": plogp.sum(1), "alt_logprob": top})
            continue
        if c["op"] == "score_grad":
            g = torch.where(have, s["d_logprob"][rows].double(), 0.0)
            hot = torch.zeros_like(p).scatter_add_(1, torch.where(have, tok, 0), g)
            d = hot - p * g.sum(1, keepdim=True)
            if c["entropy"]:
                H = plogp.sum(1, keepdim=True)
                d += (plogp - p * H) * s["d_entropy"][rows].double()[:, None]
            outs.append({"grad": torch.where(empty[:, None], 0.0, d / tau)})
            continue
        ids, score = s["teacher_tok"][rows].long(), s["teacher_score"][rows].double()
        have = ids >= 0
        lp = torch.where(have, torch.gather(logp, 1, torch.where(have, ids, 0)), 0.0)
        hot = torch.zeros_like(p, dtype=torch.bool)
        spot = torch.nn.functional.pad(hot, (0, 1))  # a column for the empty slots
        spot.scatter_(1, torch.where(have, ids, c["V"] + 1), True)
        hot = spot[:, :-1]
        if c["tail"]:
            q = torch.where(have, torch.exp(score), 0.0)
            loss = torch.where(q > 0, q * (score - lp), 0.0).sum(1)
            rest = (1 - q.sum(1)).clamp(min=0)
            left = torch.where(hot, 0.0, p).sum(1)
            loss = loss + torch.where(rest > 0, rest * (rest.log() - left.log()), 0.0)
            others = torch.where(rest > 0, rest / left, 0.0)[:, None]
            total = (q.sum(1) + rest)[:, None]
            d = torch.where(hot | (p == 0), total * p, p * (total - others))
        else:
            some = have.any(1, keepdim=True)
            logq = torch.log_softmax(torch.where(have | ~some, score / tau, NEG), dim=1)
            q = torch.where(have, logq.exp(), 0.0)
            loss = torch.where(q > 0, q * (logq - lp), 0.0).sum(1)
            d = p * some
        pulls = torch.zeros_like(p).scatter_add_(1, torch.where(have, ids, 0),
                                                 torch.where(have, q, 0.0))
        d = torch.where(empty[:, None], 0.0, d - pulls) / tau
        if s["weight"] is not None:
            w = s["weight"][rows].double()
            loss = torch.where(w != 0, loss * w, 0.0)
            d = torch.where(w[:, None] != 0, d * w[:, None], 0.0)
        outs.append({"loss": loss, "grad": d} if c["op"] == "distill_grad" else {"loss": loss})
    whole = {k: torch.cat([o[k] for o in outs]) for k in outs[0]}
    if c["op"] == "score":
        whole["alt"] = None
        whole["alt_logprob"] = whole["alt_logprob"] if c["alts"] else None
    return whole

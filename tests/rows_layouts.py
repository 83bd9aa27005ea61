"""Layouts of the row operators: for each type one width and number of rows that
takes it, at the ends of what its registers hold and of the numbers of rows for
which it is chosen; and the rows that the layouts are run on.

A call's rows are eight different ones over and over, so that every row is
compared with a float64 form of which only eight are computed. Rows lie three
values apart: at every alignment."""

import math

import numpy as np
import torch

from tests import rows_reference as R

F32, BF16 = torch.float32, torch.bfloat16
NEG = -math.inf
BASE = 8

# (waves, pieces, whether rows are cut): (values, rows) that take it
READ = {
    F32: {(1, 1, False): [(259, 1000)], (1, 2, False): [(515, 999)], (1, 4, False): [(1027, 700)],
          (1, 8, False): [(2051, 600)], (1, 16, False): [(4099, 1100)],
          (2, 16, False): [(4100, 1024), (8195, 1030)],
          (4, 8, False): [(4100, 512), (8195, 1023)],
          (4, 16, False): [(8196, 512), (16387, 600)],
          (16, 4, False): [(4100, 511), (16387, 70)],
          (16, 8, False): [(16388, 512), (32771, 65)],
          (16, 16, False): [(32772, 300), (65539, 512)],
          (4, 8, True): [(65540, 512), (140001, 70)],
          (4, 16, True): [(16388, 513), (131073, 520)]},
    BF16: {(1, 1, False): [(519, 1000)], (1, 2, False): [(1031, 999)],
           (1, 4, False): [(2055, 700)], (1, 8, False): [(4103, 600)],
           (1, 16, False): [(8199, 1100)],
           (2, 16, False): [(8200, 1024), (16391, 1030)],
           (4, 8, False): [(8200, 512), (16391, 1023)],
           (4, 16, False): [(16392, 512), (32775, 600)],
           (16, 4, False): [(8200, 511), (32775, 70)],
           (16, 8, False): [(32776, 512), (65543, 65)],
           (4, 8, True): [(65544, 512), (140001, 70)],
           (4, 16, True): [(32776, 513), (131079, 520)]},
}
# with a gradient: where it differs
GRAD = {
    F32: {**READ[F32], (16, 8, False): [(16388, 513), (32771, 65)],
          (16, 16, False): [(32772, 300), (65539, 513)],
          (4, 16, True): [(65540, 513), (131073, 520)]},
    BF16: {**READ[BF16], (16, 8, False): [(32776, 513), (65543, 65)],
           (16, 16, False): [(65544, 300), (131079, 65)],
           (4, 8, True): [(131079, 64), (131080, 512)],
           (4, 16, True): [(131080, 513), (200001, 520)]},
}


def cases(table):
    return [(d, layout, C, n) for d in table for layout, at in table[d].items() for C, n in at]


def name(p):
    if isinstance(p, torch.dtype):
        return "f32" if p == F32 else "bf16"
    return "x".join(map(str, p[:2])) + ("cut" if p[2] else "") if isinstance(p, tuple) else str(p)


def base(dtype, C, seed):
    """Eight rows: ordinary ones, masked ones, few different values, none."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((BASE, C), generator=g) * 2
    z[torch.arange(BASE), torch.randint(0, C, (BASE,), generator=g)] += 6.0
    few = torch.rand((2, C), generator=g) < 20 / C
    few[:, C // 3] = True
    z[2] = torch.where(few[0], z[2], NEG)
    z[3] = torch.where(few[1], z[3], torch.finfo(dtype).min)
    z[4] = torch.randint(0, 4, (C,), generator=g).float()  # too many candidates
    z[5] = NEG
    z[6] = torch.arange(C).float() * (6.0 / C) + 100.0  # ascending, far from zero
    return z.to(dtype), g


def rows(z, n):
    """n rows on the device, three values apart, over and over."""
    C = z.shape[1]
    buf = torch.full((n, C + 3), 55.0, dtype=z.dtype, device="cuda")
    buf[:, :C] = over(z.cuda(), n)
    return buf[:, :C], buf


def over(x, n):
    return x.repeat(-(-n // BASE), *[1] * (x.dim() - 1))[:n].contiguous()


def compare(got, want, tol):
    """Every row of got [n, ...] with that of want [8, ...]."""
    want, tol = (torch.as_tensor(np.asarray(x, np.float64)).cuda() for x in (want, tol))
    step = max(BASE, (1 << 24) // max(1, want[0].numel()) // BASE * BASE)
    for a in range(0, got.shape[0], step):
        part = got[a:a + step].double()
        w, t = over(want, part.shape[0]), over(tol, part.shape[0])
        same = (part == w) | (part.isnan() & w.isnan())
        ok = same | ((part - w).abs() <= t)
        if not bool(ok.all()):
            at = (~ok).nonzero()[:3]
            raise AssertionError([(a + int(i[0]), i[1:].tolist(), float(part[tuple(i)]),
                                   float(w[tuple(i)])) for i in at])


# ---- tolerances: those of the float32 forms (tests/test_gpu_rows.py)

SUM, REL = 1e-5, 3e-7


def check_scores(dtype, C, n):
    from paper_2608_21343_amd import capi
    z8, g = base(dtype, C, C + n)
    z, _ = rows(z8, n)
    zh = z8.float().numpy()
    tok = torch.randint(0, C, (BASE, 3), generator=g, dtype=torch.int32)
    tok[:, 0] = z8.float().argmax(1)
    tok[1, 2] = -1
    for J, M in ((3, 8), (0, 40), (1, 0)):
        t = tok[:, :J].contiguous()
        lp, lse, ent, alt_lp = (torch.full(s, 77.0, device="cuda")
                                for s in ((n, J), (n,), (n,), (n, M)))
        alt = torch.full((n, M), 77, dtype=torch.int32, device="cuda")
        capi.tb_token_logprobs(z, over(t, n).cuda() if J else None, lp if J else None, lse, ent,
                               alt if M else None, alt_lp if M else None)
        want = R.scores(zh, 1.0, t.numpy(), M)
        # a value has its own size's roundings; infinite ones have to be equal
        for got, w, tol in ((lp, want[0], SUM), (lse, want[1], SUM), (ent, want[2], 3e-5),
                            (alt_lp, want[4], SUM)):
            compare(got, w, tol + REL * np.where(np.isfinite(w), np.abs(w), 0.0))
        compare(alt, want[3], np.zeros(want[3].shape))


def check_grad(dtype, C, n):
    from paper_2608_21343_amd import capi
    z8, g = base(dtype, C, C + n + 1)
    zh = z8.float().numpy()
    tok = torch.randint(0, C, (BASE, 6), generator=g, dtype=torch.int32)
    tok[0, 5] = tok[0, 0]
    tok[1, 2] = -1
    d = torch.randn((BASE, 6), generator=g)
    d_lse, d_ent = torch.randn(BASE, generator=g), torch.randn(BASE, generator=g)
    d[7], d_lse[7], d_ent[7] = 0.0, 0.0, 0.0
    for J, ent, in_place in ((6, True, True), (2, False, False)):
        z, buf = rows(z8, n)
        t, dj = tok[:, :J].contiguous(), d[:, :J].contiguous()
        de = d_ent if ent else None
        out, room = (z, buf) if in_place else rows(torch.zeros_like(z8), n)
        capi.tb_token_logprobs_grad(z, over(t, n).cuda(), over(dj, n).cuda(), out,
                                    d_lse=over(d_lse, n).cuda(),
                                    d_entropy=over(de, n).cuda() if ent else None)
        want = R.score_grad(zh, 1.0, t.numpy(), dj.numpy(), d_lse.numpy(),
                            de.numpy() if ent else None)
        size = np.zeros((BASE, C))
        for i in range(BASE):
            logp, lse = R.softmax_row(zh[i], 1.0)
            if lse == NEG:
                continue
            p = np.exp(logp)
            size[i] = p * (abs(float(d_lse[i])) + float(dj[i].abs().sum()))
            if ent:
                size[i] += p * abs(float(d_ent[i])) * (
                    np.abs(np.where(p > 0, logp, 0.0)) + R.entropy_row(logp))
            for v, x in zip(t[i].tolist(), dj[i].tolist()):
                if v >= 0:
                    size[i, v] += abs(x)
        one = 2.0 ** -7.99 if dtype == BF16 else REL
        compare(out, want, SUM * size + 1e-37 + one * np.abs(want))
        assert bool((room[:, C:] == 55.0).all())


def check_distill(dtype, C, n, tail, grad=True):
    from paper_2608_21343_amd import capi
    z8, g = base(dtype, C, C + n + 2)
    zh = z8.float().numpy()
    K = 9
    ids = torch.randint(0, C, (BASE, K), generator=g, dtype=torch.int32)
    ids[0, 8] = ids[0, 1]
    ids[1, 4:] = -1
    # on masked rows the list names visible tokens; others stay outside it
    for i in (2, 3):
        seen = (z8[i] > -1e30).nonzero()[:, 0]
        ids[i, 0] = seen[0]
        ids[i, 1:] = -1
    sc = torch.log_softmax(torch.randn((BASE, K), generator=g), 1) - 0.4
    w = torch.tensor([1.0, 0.5, 2.0, 1.0, 3.0, 1.0, 0.25, 0.0])
    z, _ = rows(z8, n)
    loss = torch.full((n,), 77.0, device="cuda")
    out, room = rows(torch.zeros_like(z8), n)
    args = (over(ids, n).cuda(), over(sc, n).cuda(), loss)
    kw = dict(weight=over(w, n).cuda(), tail=tail, temperature=1.0 if tail else 1.5)
    tau = kw["temperature"]
    capi.tb_distill(z, *args, out if grad else None, **kw)
    want, dwant, p_rest = R.distill(zh, tau, ids.numpy(), sc.numpy().astype(np.float64), tail,
                                    w.numpy())
    with np.errstate(divide="ignore", invalid="ignore"):
        far = np.abs(np.log(np.where(p_rest > 0, p_rest, 1.0))) if tail else np.zeros(BASE)
    tol = w.numpy() * (SUM + 2e-5 + 1e-6 * (20 + far))
    tol = tol + 1e-6 * np.where(np.isfinite(want), np.abs(want), 0.0)
    compare(loss, want, tol)
    if not grad:
        return
    size = np.zeros((BASE, C))
    for i in range(BASE):
        used, q, _, mass, rest = R.teacher_row(ids.numpy()[i], sc.numpy()[i].astype(np.float64),
                                               tau, tail, C)
        logp, lse = R.softmax_row(zh[i], tau)
        if lse == NEG:
            continue
        extra = (rest + 0.1) / p_rest[i] if tail and rest > 0 and p_rest[i] > 0 else 0.0
        size[i] = np.exp(logp) * (1 + extra)
        for (v, _), qk in zip(used, q):
            size[i, v] += qk
    size *= (w.numpy() / tau)[:, None]
    one = 2.0 ** -7.99 if dtype == BF16 else REL
    tol = SUM * size + 1e-37 + one * np.abs(dwant)
    compare(out, dwant, tol)
    assert bool((room[:, C:] == 55.0).all())
    # over the logits, from the same loss
    more, room = rows(z8, n)
    capi.tb_distill(more, *args, more, **kw)
    compare(more, dwant, tol)
    assert bool((room[:, C:] == 55.0).all())

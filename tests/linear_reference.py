"""The output layer's cross entropy in float64, and how far float32 sums and the
roundings that the interface states may be from it. Plain torch on any device."""

import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step, relative


def forward(x, w, target, bias=None, weight=None):
    """(loss, lse, logits) of float64 rows; rows left out have 0."""
    z = x @ w.t()
    if bias is not None:
        z = z + bias
    lse = torch.logsumexp(z, 1)
    used = target != -1
    if weight is not None:
        used = used & (weight != 0)
    ok = (target >= 0) & (target < z.shape[1])
    hit = torch.gather(z, 1, torch.where(ok, target, 0).long()[:, None])[:, 0]
    hit = torch.where(ok, hit, math.nan)
    nll = torch.where(lse == -math.inf, math.inf, lse - hit)
    nll = torch.where(ok, nll, math.nan)
    if weight is not None:
        nll = nll * weight
    return torch.where(used, nll, 0.0), torch.where(used, lse, 0.0), z


def logit_grad(z, lse, target, weight=None, d_loss=None, d_lse=None):
    """G of the rows."""
    n = z.shape[0]
    one = torch.ones(n, dtype=z.dtype, device=z.device)
    b = one if weight is None else weight
    used = (target != -1) & (b != 0)
    b = b if d_loss is None else b * d_loss
    a = b if d_lse is None else b + d_lse
    ok = (target >= 0) & (target < z.shape[1])
    empty = lse == -math.inf
    p = torch.exp(z - torch.where(empty, 0.0, lse)[:, None])
    hot = torch.zeros_like(z).scatter_(1, torch.where(ok, target, 0).long()[:, None], 1.0)
    G = a[:, None] * p - b[:, None] * hot
    G = torch.where(ok[:, None], G, math.nan)
    used = used & ~(empty & ok) & ((a != 0) | (b != 0))
    return torch.where(used[:, None], G, 0.0)


def case(n, D, C, dtype, seed=0, bias=True, weighted=False, gaps=False, device="cpu", pad=0):
    g = torch.Generator().manual_seed(seed)

    def normal(*s):
        return torch.randn(s, generator=g)

    w = (normal(C, D) * (2.0 / math.sqrt(D))).to(dtype)
    target = torch.randint(0, C, (n,), generator=g)
    x = torch.zeros((n, D + pad), dtype=dtype)
    x[:, :D] = torch.tanh(normal(n, D) + w[target].float())
    x[:, D:] = math.nan
    if gaps:
        target[torch.rand(n, generator=g) < 0.2] = -1
    out = dict(x=x.to(device)[:, :D], w=w.to(device), target=target.to(torch.int32).to(device),
               bias=normal(C).to(dtype).to(device) if bias else None, weight=None)
    if weighted:
        weight = torch.rand(n, generator=g)
        weight[torch.rand(n, generator=g) < 0.2] = 0.0
        out["weight"] = weight.to(device)
    return out


def expected(c, d_loss=None, d_lse=None):
    """{name: (value, tolerance)} of a case's outputs.

    Sums of k float32 products in any order are off by at most (k + 9) u of the sum of
    their sizes (u = 2^-24; 8 for the planes of float32 operands, which lose up to 2^-23
    of each factor and 2^-22 of the product, and 1 for the bias). A logit
    that is off by e makes exp(z - lse) off by a factor of at most 1 + 4 e, and
    exponential, its argument and lse by another 2^-20 (arguments below 2^7 in units of
    log 2, half a step each). G is rounded to the type of the operands; the outputs
    once more."""
    u = 2.0 ** -24
    x, w = c["x"].double(), c["w"].double()
    bias = None if c["bias"] is None else c["bias"].double()
    weight = None if c["weight"] is None else c["weight"].double()
    d_loss = None if d_loss is None else d_loss.double()
    d_lse = None if d_lse is None else d_lse.double()
    dtype = c["x"].dtype
    used = c["target"] != -1
    if weight is not None:
        used = used & (weight != 0)
    x = torch.where(used[:, None], x, 0.0)  # what the others hold reaches nothing
    loss, lse, z = forward(x, w, c["target"], bias, weight)
    D, (C, n) = x.shape[1], (w.shape[0], x.shape[0])
    # (tokens that the bias masks have p = 0 whatever is added)
    big = x.abs() @ w.abs().t()
    if bias is not None:
        big = big + torch.where(bias > -1e30, bias.abs(), 0.0)
    ez = (D + 9) * u * big.amax(1)
    ok = (c["target"] >= 0) & (c["target"] < C)
    at = torch.where(ok, c["target"], 0).long()[:, None]
    hit = torch.gather(z, 1, at)[:, 0]
    tol_lse = ez + 2.0 ** -20 + 4 * u * lse.abs()
    tol_loss = 2 * ez + 2.0 ** -20 + 4 * u * (lse.abs() + hit.abs())
    if weight is not None:
        tol_loss = tol_loss * weight.abs()
    G = logit_grad(z, lse, c["target"], weight, d_loss, d_lse)
    hot = torch.zeros_like(z).scatter_(1, at, 1.0)
    a = b = torch.ones(n, dtype=z.dtype, device=z.device) if weight is None else weight.abs()
    b = b if d_loss is None else b * d_loss.abs()
    a = b if d_lse is None else b + d_lse.abs()
    p = torch.where(used[:, None], torch.exp(z - lse[:, None]), 0.0) * a[:, None]
    hot = hot * b[:, None]
    eG = p * (8 * ez[:, None] + 2.0 ** -19) + 8 * u * (p + hot)
    db_tol = eG.sum(0) + (n + 8) * u * (p + hot).sum(0)
    eG = eG + U[dtype] * G.abs() * (1 if dtype == torch.bfloat16 else 4)
    out = {"loss": (loss, tol_loss), "lse": (lse, tol_lse)}
    for name, value, size, e in (
            ("dx", G @ w, (C + 8) * u * (G.abs() @ w.abs()), eG @ w.abs()),
            ("dw", G.t() @ x, (n + 8) * u * (G.abs().t() @ x.abs()), eG.t() @ x.abs()),
            ("db", G.sum(0), db_tol, 0)):
        out[name] = (value, size + e + U[dtype] * (value.abs() + size + e) + 1e-37)
    return out


def check(got, want, name):
    value, tol = want
    got = got.double().to(value.device)
    assert got.shape == value.shape, (name, got.shape, value.shape)
    nan = torch.isnan(value)
    assert bool((torch.isnan(got) == nan).all()), f"{name}: NaN in other places"
    inf = torch.isinf(value)
    assert bool((got[inf] == value[inf]).all()), f"{name}: infinities"
    fine = ~nan & ~inf
    off = (got - value).abs()[fine]
    tol = tol.expand_as(value)[fine]
    worst = float(torch.where(off > 0, off / tol, 0.0).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{name}: off by {worst} times the tolerance"

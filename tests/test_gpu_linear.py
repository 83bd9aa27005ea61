"""The output layer's cross entropy on the GPU against float64: sizes around the
tiles, strides, rows that are left out, masked tokens, bad values, streams, graphs."""

import math

import pytest
import torch

from tests import linear_reference as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def outputs(c, names=("dx", "dw", "db")):
    x, w = c["x"], c["w"]
    made = {"dx": torch.full(x.shape, 7.0, dtype=x.dtype, device=x.device),
            "dw": torch.full(w.shape, 7.0, dtype=w.dtype, device=w.device),
            "db": torch.full((w.shape[0],), 7.0, dtype=w.dtype, device=w.device)}
    return {k: v for k, v in made.items() if k in names}


def step(c, names=("dx", "dw", "db"), **more):
    from paper_2608_21343_amd import capi
    loss, lse = torch.full((2, c["x"].shape[0]), 7.0, device="cuda")
    out = outputs(c, names)
    capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, lse, **out, bias=c["bias"],
                        weight=c["weight"], **more)
    return dict(out, loss=loss, lse=lse)


def grad(c, lse, d_loss, d_lse, names=("dx", "dw", "db")):
    from paper_2608_21343_amd import capi
    out = outputs(c, names)
    capi.tb_linear_xent_grad(c["x"], c["w"], c["target"], lse, d_loss, d_lse, **out,
                             bias=c["bias"], weight=c["weight"])
    return out


def check_all(got, want):
    for name, value in got.items():
        R.check(value, want[name], name)


SIZES = [  # rows, width, V + 1
    (1, 1, 2), (1, 64, 300), (2, 3, 255), (3, 63, 256), (5, 65, 257), (16, 64, 1025),
    (17, 128, 513), (33, 320, 999), (64, 256, 2050), (65, 200, 128), (127, 640, 129),
    (128, 129, 1025), (255, 64, 511), (256, 72, 512), (257, 333, 612), (300, 1000, 70),
    (700, 192, 3), (1025, 512, 1025), (2100, 96, 130), (40, 2048, 4099),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, D, C", SIZES)
def test_sizes(n, D, C, dtype):
    """Loss, log-sum-exp and the gradients, in one call and in two, with weights
    and rows left out in every other case."""
    some = (n + D + C) % 2 == 0
    c = R.case(n, D, C, dtype, n + C, bias=C % 3 != 0, weighted=some, gaps=some, device="cuda",
               pad=n % 3)
    want = R.expected(c)
    got = step(c)
    check_all(got, want)
    check_all(step(c, ()), {k: want[k] for k in ("loss", "lse")})
    g = torch.Generator().manual_seed(n)
    d_loss, d_lse = (torch.randn((2, n), generator=g) * 0.5).cuda()
    check_all(grad(c, got["lse"], d_loss, d_lse), R.expected(c, d_loss, d_lse))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pieces_of_the_vocabulary(dtype):
    """More gradients of logits than one piece holds."""
    from paper_2608_21343_amd import capi
    n, D, C = (6000, 64, 45001) if dtype == BF16 else (3000, 64, 30001)
    c = R.case(n, D, C, dtype, 5, device="cuda", gaps=True)
    assert capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7) < n * C * 2 * (
        1 if dtype == BF16 else 3)
    check_all(step(c), R.expected(c))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("names", [("dx",), ("dw",), ("db",), ("dw", "db")])
def test_some_gradients(names, dtype):
    c = R.case(70, 100, 600, dtype, 3, device="cuda", weighted=True)
    whole = step(c)
    some = step(c, names)
    assert set(some) == {"loss", "lse", *names}
    for name in some:
        assert bool((some[name] == whole[name]).all()), name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    """Rows of x, w, dx and dw at strides of their own; what lies between is left."""
    from paper_2608_21343_amd import capi
    for n, D, C, pads in ((40, 64, 300, (8, 16, 3, 5)), (40, 64, 300, (1, 0, 0, 64)),
                          (9, 50, 77, (0, 3, 8, 1))):
        c = R.case(n, D, C, dtype, 4, device="cuda")

        def wide(t, pad):
            buf = torch.full((t.shape[0], D + pad), math.nan, dtype=dtype, device="cuda")
            buf[:, :D] = t
            return buf[:, :D]

        c["x"], c["w"] = wide(c["x"], pads[0]), wide(c["w"], pads[1])
        want = R.expected(c)
        dx, dw = (torch.full((m, D + p), 5.0, dtype=dtype, device="cuda")
                  for m, p in ((n, pads[2]), (C, pads[3])))
        loss = torch.empty(n, device="cuda")
        capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, None, dx[:, :D], dw[:, :D],
                            bias=c["bias"])
        check_all({"loss": loss, "dx": dx[:, :D], "dw": dw[:, :D]}, want)
        assert bool((dx[:, D:] == 5).all()) and bool((dw[:, D:] == 5).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_misaligned_weights(dtype):
    n, D, C = 20, 64, 300
    c = R.case(n, D, C, dtype, 4, device="cuda")
    for name in ("x", "w"):
        buf = torch.empty(c[name].numel() + 1, dtype=dtype, device="cuda")[1:]
        c[name] = buf.view(c[name].shape).copy_(c[name])
    check_all(step(c), R.expected(c))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_left_out_hold_anything(dtype):
    c = R.case(50, 96, 400, dtype, 6, device="cuda", weighted=True, gaps=True)
    clean = step(c)
    left = (c["target"] == -1) | (c["weight"] == 0)
    assert bool(left.any())
    for value in (math.nan, math.inf, 3e38):
        c["x"][left] = value
        got = step(c)
        for name in got:
            assert bool((got[name] == clean[name]).all()), name
        assert not got["dx"][left].any() and not got["lse"][left].any()
    # their gradients reach nothing either
    clean = grad(c, clean["lse"], torch.ones(50, device="cuda"), None)
    got = grad(c, got["lse"], torch.where(left, math.nan, 1.0), None)
    for name in got:
        assert bool((got[name] == clean[name]).all()), name


def test_no_row_is_left():
    for n in (0, 1, 300):
        c = R.case(n, 64, 300, BF16, 6, device="cuda")
        c["target"][:] = -1
        got = step(c)
        for name, value in got.items():
            assert not value.any(), name
        got = grad(c, torch.zeros(n, device="cuda"), None, None)
        assert not got["dx"].any() and not got["dw"].any() and not got["db"].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_targets_out_of_range(dtype):
    c = R.case(40, 64, 300, dtype, 8, device="cuda")
    c["target"][3], c["target"][17], c["target"][20] = 300, -2, 2 ** 31 - 1
    got = step(c)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 17, 20]] = True
    assert bool((torch.isnan(got["loss"]) == bad).all())
    assert bool(torch.isfinite(got["lse"]).all())
    assert bool((torch.isnan(got["dx"]).all(1) == bad).all())
    assert bool((torch.isnan(got["dx"]).any(1) == bad).all())
    assert bool(torch.isnan(got["dw"]).all()) and bool(torch.isnan(got["db"]).all())
    R.check(got["lse"], R.expected(c)["lse"], "lse")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_tokens(dtype):
    """Tokens whose bias is -inf or the lowest value, a target among them, and a
    layer in which all are."""
    c = R.case(30, 64, 520, dtype, 9, device="cuda")
    c["bias"][40:500] = -math.inf
    c["bias"][500:510] = torch.finfo(dtype).min
    c["target"] %= 40
    want = R.expected(c)
    check_all(step(c), want)
    c["target"][5] = 100
    got = step(c)
    assert got["loss"][5] == math.inf and not torch.isinf(got["loss"]).sum() > 1
    assert bool(torch.isfinite(got["dx"]).all())
    # the masked target is pulled all the same: G is p - 1 there
    G_t = got["db"][100].item()
    assert abs(G_t + 1) <= 2.0 ** -8
    c["bias"][:] = -math.inf
    got = step(c)
    assert bool((got["loss"] == math.inf).all()) and bool((got["lse"] == -math.inf).all())
    assert not got["dx"].any() and not got["dw"].any() and not got["db"].any()
    two = grad(c, got["lse"], None, None)
    assert not two["dx"].any() and not two["dw"].any() and not two["db"].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_bad_values_stay_in_their_rows(dtype, value):
    c = R.case(300, 64, 600, dtype, 10, device="cuda")
    clean = step(c)
    c["x"][[7, 290], 5] = value
    got = step(c)
    bad = torch.zeros(300, dtype=torch.bool, device="cuda")
    bad[[7, 290]] = True
    for name in ("loss", "lse"):
        assert bool((torch.isnan(got[name]) == bad).all()), name
        assert bool((got[name][~bad] == clean[name][~bad]).all()), name
    assert bool(torch.isnan(got["dx"][bad]).all())
    assert bool((got["dx"][~bad] == clean["dx"][~bad]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_other_sizes(dtype):
    """A row of large features, one of tiny ones and rows of very different weights
    are as good as if they were alone."""
    c = R.case(40, 64, 300, dtype, 11, device="cuda", weighted=True)
    c["x"][3] *= 1e4
    c["x"][4] *= 1e-20
    c["weight"][5:9] = torch.tensor([1e-20, 1e20, 1e-3, 1e3])
    want = R.expected(c)
    got = step(c)
    for name in ("loss", "lse", "dx", "dw", "db"):
        R.check(got[name], want[name], name)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinite_and_nan_weights(dtype):
    c = R.case(40, 64, 300, dtype, 11, device="cuda", weighted=True)
    c["weight"][:] = 0.5
    clean = step(c)
    for value in (math.inf, math.nan):
        c["weight"][6] = value
        got = step(c)
        others = torch.arange(40, device="cuda") != 6
        assert bool((got["dx"][others] == clean["dx"][others]).all())
        assert bool((got["loss"][others] == clean["loss"][others]).all())
        assert not bool(torch.isfinite(got["dx"][6]).any())
        assert bool(torch.isfinite(got["lse"]).all())


def test_results_repeat():
    """The same bits again, also with other work on the card and other workspace
    contents."""
    from paper_2608_21343_amd import capi
    c = R.case(1500, 256, 1025, BF16, 12, device="cuda", weighted=True, gaps=True)
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7)
    first = step(c)
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        again = step(c, workspace=ws)
        for name in first:
            assert bool((first[name] == again[name]).all()), name


def test_workspace_too_small():
    from paper_2608_21343_amd import capi
    c = R.case(20, 64, 300, BF16, 1, device="cuda")
    need = capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7)
    ws = torch.empty(need - 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(capi.TbError, match="needs"):
        step(c, workspace=ws)


def test_other_stream():
    from paper_2608_21343_amd import capi
    c = R.case(200, 256, 1025, BF16, 2, device="cuda")
    want = step(c)
    side = torch.cuda.Stream()
    out = outputs(c)
    loss = torch.empty(200, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        capi.tb_linear_xent(c["x"], c["w"], c["target"], loss, None, **out, bias=c["bias"],
                            stream=side)
        # memory that the call's workspace must not share
        junk = [torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    del junk
    for name in out:
        assert bool((out[name] == want[name]).all()), name
    assert bool((loss == want["loss"]).all())


def test_two_graphs_of_one_workspace():
    """Captured calls that share a workspace, replayed in turns with eager work between."""
    from paper_2608_21343_amd import capi
    cases = [R.case(n, 64, C, BF16, 3, device="cuda", gaps=True) for n, C in ((90, 700), (300, 333))]
    want = [step(c) for c in cases]
    need = max(capi.tb_linear_xent_workspace_bytes(c["x"], c["w"], 7) for c in cases)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for c in cases:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(c, workspace=ws)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(c, workspace=ws))
        graphs.append(graph)
    for turn in range(3):
        for graph, out, right in zip(graphs, outs, want):
            for value in out.values():
                value.fill_(3.0)
            ws.fill_(turn * 100)
            graph.replay()
            torch.cuda.synchronize()
            for name in out:
                assert bool((out[name] == right[name]).all()), name


# ---- autograd


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_autograd_layer(dtype):
    """loss and lse in a larger expression, over leading dimensions."""
    from paper_2608_21343_amd.linearops import linear_xent
    c = R.case(60, 96, 400, dtype, 13, device="cuda", weighted=True, gaps=True)
    leaves = [c[k].detach().clone().requires_grad_() for k in ("x", "w", "bias")]
    x = leaves[0].view(3, 20, 96)
    out = linear_xent(x, leaves[1], c["target"].view(3, 20), leaves[2], c["weight"].view(3, 20))
    assert out.loss.shape == out.lse.shape == (3, 20)
    (out.loss.sum() * 2 + 1e-2 * out.lse.square().sum()).backward()
    lse = out.lse.detach().flatten()
    want = R.expected(c, torch.full_like(lse, 2.0), 2e-2 * lse)
    for leaf, name in zip(leaves, ("dx", "dw", "db")):
        R.check(leaf.grad, want[name], name)


def test_autograd_against_differences():
    """Central differences of the kernel's own loss along one direction. Their error:
    the loss's rounding 2 * tolerance / 2h, and h^2 / 6 of a third derivative, which for a
    log-sum-exp is at most (2 max |dz|)^3 a row."""
    from paper_2608_21343_amd.linearops import linear_xent
    c = R.case(40, 64, 200, F32, 14, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    move = {k: torch.randn(c[k].shape, generator=g, device="cuda") * 0.1 for k in ("x", "w", "bias")}
    leaves = {k: c[k].clone().requires_grad_() for k in move}
    grads = torch.autograd.grad(linear_xent(leaves["x"], leaves["w"], c["target"],
                                            leaves["bias"]).loss.sum(), list(leaves.values()))
    slope = sum(float((a.double() * b.double()).sum()) for a, b in zip(grads, move.values()))
    h = 2.0 ** -4

    def at(t):
        moved = {k: c[k] + t * move[k] for k in move}
        return linear_xent(moved["x"], moved["w"], c["target"], moved["bias"]).loss.double().sum()

    got = float(at(h) - at(-h)) / (2 * h)
    X, W = c["x"].double(), c["w"].double()
    dX, dW = move["x"].double(), move["w"].double()
    dz = (dX.abs() @ W.abs().t() + X.abs() @ dW.abs().t() + 2 * h * dX.abs() @ dW.abs().t()
          + move["bias"].double().abs()).amax(1)
    # z itself is quadratic in t: its second derivative, and its product with the first
    ddz = 2 * (dX.abs() @ dW.abs().t()).amax(1)
    third = ((2 * dz) ** 3 + 3 * (2 * dz) * 2 * ddz).sum()
    rounding = R.expected(c)["loss"][1].sum() * 1.5
    assert abs(got - slope) <= float(third) * h * h / 6 + float(rounding) / h


def test_autograd_of_some_leaves_and_views():
    from paper_2608_21343_amd.linearops import linear_xent, linear_xent_step
    c = R.case(24, 64, 100, F32, 15, device="cuda")
    want = R.expected(c)
    w = c["w"].t().contiguous().t().requires_grad_()  # columns first: copied
    loss = linear_xent(c["x"], w, c["target"], c["bias"]).loss
    loss.sum().backward()
    R.check(w.grad, want["dw"], "dw")
    # a broadcast row of features
    one = c["x"][:1].clone().requires_grad_()
    loss = linear_xent(one.expand(24, 64), c["w"], c["target"], c["bias"]).loss
    loss.sum().backward()
    d = dict(c, x=c["x"][:1].expand(24, 64))
    value, tol = R.expected(d)["dx"]
    R.check(one.grad[0], (value.sum(0), tol.sum(0) + 24 * 2.0 ** -23 * value.abs().sum(0)), "dx")
    loss, dx, dw, db = linear_xent_step(c["x"].expand(1, 24, 64), c["w"], c["target"][None],
                                        c["bias"])
    check_all({"loss": loss[0], "dx": dx[0], "dw": dw, "db": db}, want)
    assert linear_xent_step(c["x"], c["w"], c["target"])[3] is None


def test_autograd_refusals():
    from paper_2608_21343_amd.linearops import linear_xent
    c = R.case(24, 64, 100, F32, 15, device="cuda")
    weight = torch.ones(24, device="cuda")
    with pytest.raises(ValueError, match="weight"):
        linear_xent(c["x"], c["w"], c["target"], weight=weight.clone().requires_grad_())
    with pytest.raises(ValueError, match="one dtype"):
        linear_xent(c["x"], c["w"].bfloat16(), c["target"])
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        linear_xent(c["x"].half(), c["w"].half(), c["target"])
    with pytest.raises(ValueError, match="target"):
        linear_xent(c["x"], c["w"], c["target"][:20])
    with pytest.raises(ValueError, match="width"):
        linear_xent(c["x"], c["w"][:, :32], c["target"])
    with pytest.raises(ValueError, match="dtype"):
        linear_xent(c["x"], c["w"], c["target"].long())
    x = c["x"].clone().requires_grad_()
    loss = linear_xent(x, c["w"], c["target"]).loss.sum()
    g, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        g.pow(2).sum().backward()
    y = x * 1.0
    loss = linear_xent(y, c["w"], c["target"]).loss.sum()
    y.detach().mul_(2.0)
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()


def test_backward_captured():
    """Forward and backward pass in a captured graph, every replay as the eager one."""
    from paper_2608_21343_amd.linearops import linear_xent
    c = R.case(100, 64, 500, BF16, 16, device="cuda")
    x, w = c["x"].clone().requires_grad_(), c["w"].clone().requires_grad_()

    def run():
        loss = linear_xent(x, w, c["target"], c["bias"]).loss.sum()
        return (loss, *torch.autograd.grad(loss, (x, w)))

    want = [t.detach().clone() for t in run()]  # (no graph of it stays)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        for t in out[1:]:
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((a == b).all()) for a, b in zip(out[1:], want[1:]))
        run()

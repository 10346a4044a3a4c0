"""fp16 gradients of the class loss where rows' g_loss differ by many orders: what only light rows contribute to keeps fp16's digits.

Rows of two groups, heavy and light, with values in columns of their own, so that g_w's light columns hold what light rows give and nothing else.
Tolerances, u = 2^-24, half = 2^-11: a logit's error `zerr`, as tests/test_gpu_class_loss.py derives it; every term G_ik x_ij of g_w with G and the row of x times its weight
rounded to fp16 once each, fp32 chains of (n / 16 + 20) steps of 2 u, an exponential near 1 minus 1 that keeps the exponential's error; then the output's half step, and
2^-25 below its normal range.  Below fp16's normal range the two factors are off by 2^-25 of a unit each.  A row whose weight is w of the largest one's W enters
as x w 2^b in [2^-6, 2^-5) |x| where w < 2^-5, b <= 18, and G as G 2^(14 - b): in g_w's units 2^-25 2^-b W |G| <= 2^-19 w W |G| (w >= 2^-24) beside a row of x, and
2^-25 2^(b - 14) w W |x| <= 2^-44 W |x| beside G."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U, HALF = 2.0 ** -24, 2.0 ** -11


@pytest.fixture(scope="module")
def ctx():
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    yield c
    c.close()


def problem(n, d, classes, light, seed, labelled=1.0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn((classes, d), device="cuda", generator=gen) / d ** 0.5).half()
    x = torch.randn((n, d + pad), device="cuda", generator=gen)
    is_light = torch.arange(n, device="cuda") % 2 == 1
    x[is_light, :d // 2] = 0
    x[~is_light, d // 2:d] = 0
    labels = torch.randint(0, classes, (n,), device="cuda", generator=gen)
    labels[torch.rand(n, device="cuda", generator=gen) >= labelled] = -1
    # scaled as a loss is that trains in fp16: gradients of light rows are normal numbers, too
    g = (torch.rand(n, device="cuda", generator=gen) + 0.5) * torch.where(is_light, light, 1.0)
    return x.half()[:, :d], W, labels, g * (2.0 ** 14 / n), is_light


def expected(x, W, labels, g):
    n, d = x.shape
    kept = torch.nonzero(labels >= 0)[:, 0]
    xd, wd, gd, y = x[kept].double(), W.double(), g[kept].double(), labels[kept]
    z = xd @ wd.t()
    zerr = (d / 16 + 4) * 2 * U * (xd.abs() @ wd.abs().t()).amax(1)
    lse = torch.logsumexp(z, 1)
    p = (z - lse[:, None]).exp()
    G = p.clone()
    G[torch.arange(y.numel(), device=y.device), y] -= 1
    top = float(gd.abs().max())
    slack = p * (3 * zerr[:, None] + 300 * U)
    off_w = G.abs() * (2 * HALF + (n / 16 + 20) * 2 * U) + slack
    gw = (G * gd[:, None]).t() @ xd
    room_w = gw.abs() * HALF + 1.01 * ((off_w * gd.abs()[:, None]).t() @ xd.abs()) + 2.0 ** -25 + 2.0 ** -19 * (G.abs() * gd.abs()[:, None]).sum(0)[:, None] \
        + 2.0 ** -44 * top * xd.abs().sum(0)
    off_x = (G.abs() * (HALF + (W.shape[0] / 16 + 20) * 2 * U) + slack) * gd.abs()[:, None] + 2.0 ** -44 * top
    gx = torch.zeros((n, d), dtype=torch.float64, device=x.device)
    room_x = torch.zeros_like(gx)
    gx[kept] = (G * gd[:, None]) @ wd
    room_x[kept] = gx[kept].abs() * HALF + 1.01 * (off_x @ wd.abs()) + 2.0 ** -25
    # rows between w = 2^-5 and 1 keep their 2^14: half a step of 2^-25 of those
    room_x[kept] += 2.0 ** -39 * gd.abs()[:, None] * wd.abs().sum(0)
    return gx, room_x, gw, room_w


@pytest.mark.parametrize("light", [1.0, 0.03, 1e-3, 1e-5, 1e-6, 2.0 ** -22])
@pytest.mark.parametrize("n,d,classes,labelled,pad", [(64, 32, 10, 1.0, 0), (300, 64, 47, 1.0, 0), (500, 130, 300, 0.7, 0), (200, 64, 40, 1.0, 3), (5000, 48, 20, 0.3, 8), (9000, 64, 130, 1.0, 0)])
def test_light_rows_keep_their_digits(ctx, n, d, classes, labelled, pad, light):
    x, W, labels, g, is_light = problem(n, d, classes, light, n + d, labelled, pad)
    _, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g)
    ctx.sync_check()
    gx, room_x, gw, room_w = expected(x, W, labels, g)
    assert ((g_x.double() - gx).abs() <= room_x).all()
    assert ((g_w.double() - gw).abs() <= room_w).all()
    # as a whole, too: three roundings to fp16 of independent terms, each at most half a step
    of_light = slice(d // 2, d)
    assert float((g_w.double() - gw)[:, of_light].norm() / gw[:, of_light].norm()) <= 3 * HALF + 2.0 ** -25 * gw[:, of_light].numel() ** 0.5 / float(gw[:, of_light].norm())


def test_each_gradient_alone_and_every_time(ctx):
    x, W, labels, g, _ = problem(700, 64, 90, 1e-5, 5, 0.8)
    _, lse = ctx.class_loss(x, W, labels)
    both = ctx.class_loss_backward(x, W, labels, lse, g)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(both, ctx.class_loss_backward(x, W, labels, lse, g)))
    assert torch.equal(ctx.class_loss_backward(x, W, labels, lse, g, want_g_w=False)[0], both[0])
    assert torch.equal(ctx.class_loss_backward(x, W, labels, lse, g, want_g_x=False)[1], both[1])
    ctx.sync_check()


def test_weights_that_are_nothing_or_not_finite(ctx):
    x, W, labels, g, _ = problem(300, 64, 47, 1e-4, 6)
    _, lse = ctx.class_loss(x, W, labels)
    some = g.clone()
    some[::3] = 0
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, some)
    ctx.sync_check()
    gx, room_x, gw, room_w = expected(x, W, labels, some)
    assert (g_x[::3] == 0).all() and ((g_x.double() - gx).abs() <= room_x).all() and ((g_w.double() - gw).abs() <= room_w).all()
    some[7] = float("nan")
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, some)
    ctx.sync_check()
    assert torch.isnan(g_x[7]).all() and torch.isnan(g_w).any()


def test_rows_of_2_to_the_minus_29_beside_results_past_fp16(ctx):
    """Heavy rows' results are infinite in fp16, light ones' ordinary numbers.  x 2^-29 2^18 is off by 2^-25 beside its half step, which is 2^-14 of values of x near 1, and G
    2^(14 - 18) by 2^-25 of at most 2^-4: with three roundings of half a step each, less than four in the 2-norm."""
    n, d, classes, light = 400, 64, 30, 2.0 ** -29
    x, W, labels, g, is_light = problem(n, d, classes, light, 8)
    g = g * 2.0 ** 16
    _, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g)
    ctx.sync_check()
    gx, _, gw, _ = expected(x, W, labels, g)
    for got, want in ((g_x[is_light], gx[is_light]), (g_w[:, d // 2:], gw[:, d // 2:])):
        assert float((got.double() - want).norm() / want.norm()) <= 4 * HALF
    assert torch.isinf(g_x[~is_light]).any() and torch.isinf(g_w[:, :d // 2]).any()


def test_captured_and_replayed():
    """The memory that holds the largest weight is cleared before the kernels that find it: within a graph, too, and again at every replay."""
    from paper_2210_13149_b200 import binding as B
    stream = torch.cuda.Stream()
    first, second = problem(5000, 48, 60, 1e-4, 9, 0.7), problem(5000, 48, 60, 1e-2, 10, 0.4)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = B.BiGCN(0)
        x, W, labels, g, _ = [t.clone() for t in first]
        _, lse = c.class_loss(x, W, labels)
        c.class_loss_backward(x, W, labels, lse, g)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            loss, lse = c.class_loss(x, W, labels)
            out = (loss, lse) + c.class_loss_backward(x, W, labels, lse, g)
        for given, factor in ((first, 1.0), (second, 1.0), (second, 2.0 ** -9), (first, 1.0)):
            for t, v in zip((x, W, labels), given):
                t.copy_(v)
            g.copy_(given[3] * factor)
            graph.replay()
            stream.synchronize()
            want = c.class_loss(x, W, labels)
            want = want + c.class_loss_backward(x, W, labels, want[1], g)
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        c.sync_check()

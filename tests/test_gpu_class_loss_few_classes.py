"""Gradients of the class loss against up to 64 classes: G keeps twice the digits of its type, so that a gradient is the exact one rounded once, also where its terms cancel.

Tolerances, u = 2^-24, half = half a step of the type (2^-8 bf16, 2^-11 fp16): a logit's error `zerr`, the exponential's (300 u) and the chains' as
tests/test_gpu_class_loss.py derives them; a term G_ik w_kj with G in two halves, each rounded: half^2 of it (the low half is at most half |G|); in fp16 the low half may be
below the normal range: 2^-25 of G's unit 2^14, and rows of x are rounded once more where weights differ; then the result's half step."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    yield c
    c.close()


def problem(n, d, classes, seed, dtype, labelled=1.0, pad=0, even=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn((classes, d + pad), device="cuda", generator=gen) / d ** 0.5).to(dtype)[:, :d]
    x = torch.randn((n, d + pad), device="cuda", generator=gen).to(dtype)[:, :d]
    labels = torch.randint(0, classes, (n,), device="cuda", generator=gen)
    labels[torch.rand(n, device="cuda", generator=gen) >= labelled] = -1
    g = torch.full((n,), 1.0 / n, device="cuda") if even else (torch.rand(n, device="cuda", generator=gen) + 0.1) / n
    return x, W, labels, g


def expected(x, W, labels, g):
    n, d = x.shape
    half = torch.finfo(x.dtype).eps / 2
    kept = torch.nonzero(labels >= 0)[:, 0]
    xd, wd, gd, y = x[kept].double(), W.double(), g[kept].double()[:, None], labels[kept]
    z = xd @ wd.t()
    zerr = (d / 16 + 4) * 2 * U * (xd.abs() @ wd.abs().t()).amax(1, keepdim=True)
    p = torch.softmax(z, 1)
    G = p.clone()
    G[torch.arange(y.numel(), device=y.device), y] -= 1
    slack = p * (3 * zerr + 300 * U)
    least = 2.0 ** -39 if x.dtype == torch.float16 else 0.0
    once_more = half if x.dtype == torch.float16 and g[kept].unique().numel() > 1 else 0.0
    terms_x = (G.abs() * (1.01 * half ** 2 + (2 * 64 / 16 + 20) * 2 * U) + slack + least) * gd
    terms_w = (G.abs() * (1.01 * half ** 2 + once_more + (2 * n / 16 + 20) * 2 * U) + slack + least) * gd
    tiny = 2.0 ** -25 if x.dtype == torch.float16 else 1e-38
    gx, room_x = torch.zeros((n, d), dtype=torch.float64, device=x.device), torch.full((n, d), tiny, dtype=torch.float64, device=x.device)
    gx[kept] = (G * gd) @ wd
    room_x[kept] += gx[kept].abs() * half + 1.01 * (terms_x @ wd.abs())
    gw = (G * gd).t() @ xd
    low = 2.0 ** -25 * float(gd.abs().max()) * G.abs().sum(0)[:, None] if once_more else 0.0
    return gx, room_x, gw, gw.abs() * half + 1.01 * (terms_w.t() @ xd.abs()) + low + tiny


@pytest.mark.parametrize("n,d,classes,labelled,pad", [(1, 1, 1, 1.0, 0), (3, 8, 2, 1.0, 0), (64, 1, 40, 1.0, 0), (300, 1, 64, 0.7, 0), (141, 64, 7, 1.0, 0), (2708, 64, 7, 0.052, 0),
                                                       (129, 100, 47, 1.0, 0), (700, 256, 64, 1.0, 0), (700, 257, 63, 0.5, 0), (400, 500, 32, 1.0, 0), (400, 130, 33, 0.6, 5), (5000, 300, 31, 0.9, 0), (5000, 48, 33, 0.3, 3), (200, 4096, 20, 1.0, 0),
                                                       (30000, 256, 47, 0.08, 0), (9000, 500, 18, 1.0, 12)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("even", [True, False])
def test_gradients_are_rounded_once(ctx, n, d, classes, labelled, pad, dtype, even):
    x, W, labels, g = problem(n, d, classes, n + d, dtype, labelled, pad, even)
    if dtype == torch.float16:
        g = g * n                               # results in fp16's normal range
    _, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g)
    ctx.sync_check()
    gx, room_x, gw, room_w = expected(x, W, labels, g)
    assert ((g_x.double() - gx).abs() <= room_x).all()
    assert ((g_w.double() - gw).abs() <= room_w).all()
    assert torch.equal(ctx.class_loss_backward(x, W, labels, lse, g, want_g_w=False)[0], g_x)
    assert torch.equal(ctx.class_loss_backward(x, W, labels, lse, g, want_g_x=False)[1], g_w)


@pytest.mark.parametrize("classes", [5, 40])
def test_rows_in_pieces(ctx, classes):
    """More rows than one piece of G holds (4,194,304): the second piece's sums are added to the first one's."""
    n, d = 4_200_000, 8
    x, W, labels, g = problem(n, d, classes, 3, torch.bfloat16)
    _, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g)
    ctx.sync_check()
    gx, room_x, gw, room_w = expected(x, W, labels, g)
    assert ((g_x.double() - gx).abs() <= room_x).all()
    assert ((g_w.double() - gw).abs() <= room_w).all()


def test_the_last_classes_of_many(ctx):
    """Classes in pieces whose last one holds fewer than 64: as the others before it, in one half."""
    n, d, classes = 20000, 32, 16384 + 40
    x, W, labels, g = problem(n, d, classes, 5, torch.bfloat16)
    _, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g)
    ctx.sync_check()
    gx, gw = torch.zeros((n, d), dtype=torch.float64, device="cuda"), torch.zeros((classes, d), dtype=torch.float64, device="cuda")
    for a in range(0, n, 4000):
        r = slice(a, a + 4000)
        G = torch.softmax(x[r].double() @ W.double().t(), 1)
        G[torch.arange(4000, device="cuda"), labels[r]] -= 1
        gx[r] = G @ W.double() / n
        gw += G.t() @ x[r].double() / n
    # two roundings of half a step each, of independent terms
    assert float((g_x.double() - gx).norm() / gx.norm()) <= 2.0 ** -8 and float((g_w.double() - gw).norm() / gw.norm()) <= 2.0 ** -8

"""Softmax cross entropy against a class matrix and its gradients, against the formulas in 64 bits.

Tolerances, u = 2^-24.  A logit is a sum of exact products that the tensor cores add in steps of 16, each cut to 2 u of the sum of
magnitudes at worst: (d / 16 + 4) 2 u of that sum, `zerr`.  The sum of exponentials adds at most 128 terms in chains, then parts of
those: 128 u, with 8 u for the exponential's own error.  G is rounded to the operands' type, half a step (e / 2) of each term of
the gradients' sums, and an exponential near 1 minus 1 keeps the exponential's absolute error; then the output's own half step."""
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


def problem(n, d, classes, seed, labelled=1.0, dtype=torch.bfloat16, pad=0, shift=0, scale=2.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = (torch.randn((classes, d + pad + shift), device="cuda", generator=gen) / d ** 0.5).to(dtype)[:, shift:shift + d]
    labels = torch.randint(0, classes, (n,), device="cuda", generator=gen)
    x = torch.randn((n, d + pad + shift), device="cuda", generator=gen) * scale
    x[:, shift:shift + d] += W[labels].float() * torch.rand((n, 1), device="cuda", generator=gen) * 8
    x = x.to(dtype)[:, shift:shift + d]
    if labelled < 1:
        labels = torch.where(torch.rand(n, device="cuda", generator=gen) < labelled, labels, torch.full_like(labels, -1))
    g_loss = torch.rand(n, device="cuda", generator=gen) / n
    return x, W, labels, g_loss


def reference(x, W, labels, g_loss):
    """loss, lse, g_x, g_w and what each may be off by, over the labelled rows; zero elsewhere."""
    n, d = x.shape
    kept = torch.nonzero(labels >= 0)[:, 0]
    xd, wd = x[kept].double(), W.double()
    z = xd @ wd.t()
    zerr = (d / 16 + 4) * 2 * U * (xd.abs() @ wd.abs().t()).amax(1) if kept.numel() else z.sum(1)
    lse = torch.logsumexp(z, 1)
    y = labels[kept]
    at = z.gather(1, y[:, None])[:, 0]
    p = (z - lse[:, None]).exp()
    one = torch.zeros_like(p)
    one[torch.arange(y.numel(), device=y.device), y] = 1
    G = (p - one) * g_loss[kept].double()[:, None]
    half = torch.finfo(x.dtype).eps / 2
    chain = (W.shape[0] / 16 + 20) * 2 * U
    off = G.abs() * (half + chain) + p * g_loss[kept].abs().double()[:, None] * (3 * zerr[:, None] + 300 * U)
    chain_w = (n / 16 + 20) * 2 * U
    once_more = half if x.dtype == torch.float16 else 0.0           # rows of x times g_loss / max |g_loss| are rounded, too
    off_w = G.abs() * (half + once_more + chain_w) + p * g_loss[kept].abs().double()[:, None] * (3 * zerr[:, None] + 300 * U)

    if x.dtype == torch.float16:                                    # 2^14 G below the normal range: half a step, 2^-25
        least = 2.0 ** -39 * g_loss[kept].abs().double()[:, None]
        off, off_w = off + least, off_w + least
    # and the rows of x, scaled, below theirs: 2^-25 of the largest weight
    low = (p - one).abs().sum(0)[:, None] * 2.0 ** -25 * g_loss[kept].abs().double().max() if x.dtype == torch.float16 and kept.numel() else 0.0

    def whole(v):
        out = torch.zeros((n,) + v.shape[1:], dtype=torch.float64, device=x.device)
        out[kept] = v
        return out

    gx, gw = G @ wd, G.t() @ xd
    return {"loss": (whole(lse - at), whole(2 * zerr + 136 * U + 4 * U * (lse.abs() + at.abs()))),
            "lse": (whole(lse), whole(zerr + 136 * U + 4 * U * (lse.abs() + at.abs()))),
            "g_x": (whole(gx), whole(gx.abs() * half + 1.01 * off @ wd.abs())), "g_w": (gw, gw.abs() * half + 1.01 * off_w.t() @ xd.abs() + low)}


def check(ctx, x, W, labels, g_loss):
    loss, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g_loss)
    ctx.sync_check()
    ref = reference(x, W, labels, g_loss)
    tiny = 2.0 ** -24 if x.dtype == torch.float16 else 1e-38
    for name, got in (("loss", loss), ("lse", lse), ("g_x", g_x), ("g_w", g_w)):
        want, room = ref[name]
        err = (got.double() - want).abs()
        assert got.shape == want.shape and got.dtype == (torch.float32 if name in ("loss", "lse") else x.dtype)
        assert (err <= room + tiny).all(), (name, float((err - room).max()), float(want.abs().max()))
    return loss, lse, g_x, g_w


SIZES = [(1, 1, 1), (1, 8, 2), (2, 16, 3), (5, 17, 7), (1, 64, 1000), (3, 100, 30011), (7, 602, 47), (128, 64, 64), (129, 65, 65), (127, 256, 40), (140, 64, 7),
         (256, 128, 256), (257, 129, 257), (300, 500, 1000), (33, 1433, 129), (1000, 256, 47), (2708, 64, 7), (200, 4096, 300), (500, 72, 513), (64, 16384, 20)]


@pytest.mark.parametrize("n,d,classes", SIZES)
def test_loss_and_gradients(ctx, n, d, classes):
    check(ctx, *problem(n, d, classes, n + d))


@pytest.mark.parametrize("n,d,classes", SIZES)
def test_loss_and_gradients_in_fp16(ctx, n, d, classes):
    x, W, labels, g_loss = problem(n, d, classes, n + d, dtype=torch.float16)
    check(ctx, x, W, labels, torch.full_like(g_loss, 1.0 / n))
    check(ctx, x, W, labels, g_loss * torch.where(torch.arange(n, device="cuda") % 3 == 0, -1.0, 1.0))


@pytest.mark.parametrize("n,labelled,pad,shift", [(200, 0.0, 0, 0), (200, 0.5, 0, 0), (5000, 0.05, 0, 0), (6000, 0.97, 0, 0), (6000, 1.0, 0, 0), (150, 0.4, 5, 1)])
def test_fp16_rows_without_a_label(ctx, n, labelled, pad, shift):
    x, W, labels, g_loss = problem(n, 64, 300, n, labelled, dtype=torch.float16, pad=pad, shift=shift)
    out = check(ctx, x, W, labels, g_loss)
    bad = x.clone()
    bad[labels < 0] = float("nan")
    g_bad = torch.where(labels < 0, torch.full_like(g_loss, float("nan")), g_loss)
    loss, lse = ctx.class_loss(bad, W, labels)
    got = (loss, lse) + ctx.class_loss_backward(bad, W, labels, lse, g_bad)
    ctx.sync_check()
    assert all(torch.equal(a, b) for a, b in zip(out, got))


def test_fp16_with_a_gradient_of_nothing(ctx):
    x, W, labels, g_loss = problem(90, 64, 300, 3, dtype=torch.float16)
    _, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, torch.zeros_like(g_loss))
    ctx.sync_check()
    assert (g_x == 0).all() and (g_w == 0).all()


@pytest.mark.parametrize("n,d,classes", [(1, 8, 2), (5, 17, 7), (140, 64, 7), (300, 130, 260), (5000, 64, 47), (4097, 24, 5), (20000, 16, 3)])
@pytest.mark.parametrize("labelled", [0.0, 0.05, 0.5, 0.97])
def test_rows_without_a_label_take_no_part(ctx, n, d, classes, labelled):
    x, W, labels, g_loss = problem(n, d, classes, n, labelled)
    out = check(ctx, x, W, labels, g_loss)
    bad = x.clone()
    bad[labels < 0] = float("nan")
    bad[torch.nonzero(labels < 0)[::2, 0]] = float("inf")
    g_bad = torch.where(labels < 0, torch.full_like(g_loss, float("nan")), g_loss)
    loss, lse = ctx.class_loss(bad, W, labels)
    g_x, g_w = ctx.class_loss_backward(bad, W, labels, lse, g_bad)
    ctx.sync_check()
    assert all(torch.equal(a, b) for a, b in zip(out, (loss, lse, g_x, g_w)))
    skipped = labels < 0
    assert (loss[skipped] == 0).all() and (lse[skipped] == 0).all() and (g_x[skipped] == 0).all()


@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (0, 1), (3, 4), (0, 8)])
def test_rows_of_a_wider_matrix(ctx, pad, shift):
    for labelled in (1.0, 0.4):
        check(ctx, *problem(150, 100, 90, 5, labelled, pad=pad, shift=shift))


def test_a_label_that_is_no_class_shows(ctx):
    x, W, labels, g_loss = problem(50, 32, 10, 6)
    labels[7], labels[8] = 10, 2 ** 40
    loss, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g_loss)
    ctx.sync_check()
    assert torch.isnan(loss[7:9]).all() and torch.isnan(lse[7:9]).all() and (g_x[7:9] == 0).all()
    rest = torch.where(labels >= 10, torch.full_like(labels, -1), labels)
    ref = reference(x, W, rest, g_loss)
    keep = rest >= 0
    assert ((loss.double() - ref["loss"][0])[keep].abs() <= ref["loss"][1][keep]).all()
    assert ((g_w.double() - ref["g_w"][0]).abs() <= ref["g_w"][1] + 1e-38).all()


def test_a_row_that_is_not_finite_spoils_itself_and_the_class_gradient(ctx):
    x, W, labels, g_loss = problem(200, 64, 300, 7)
    want = ctx.class_loss(x, W, labels)
    bad = x.clone()
    bad[5, 3] = float("nan")
    loss, lse = ctx.class_loss(bad, W, labels)
    g_x, _ = ctx.class_loss_backward(bad, W, labels, lse, g_loss, want_g_w=False)
    ctx.sync_check()
    keep = torch.arange(200, device="cuda") != 5
    assert torch.isnan(loss[5]) and torch.isnan(lse[5]) and torch.isnan(g_x[5]).all()
    assert torch.equal(loss[keep], want[0][keep]) and torch.equal(lse[keep], want[1][keep]) and torch.isfinite(g_x[keep]).all()


def test_far_logits(ctx):
    """Logits of some hundreds: exp would overflow without the maximum; losses near 0 keep their digits."""
    x, W, labels, g_loss = problem(300, 64, 700, 8, scale=60.0)
    check(ctx, x, W, labels, g_loss)
    d, classes = 64, 500
    W = torch.zeros((classes, d), device="cuda", dtype=torch.bfloat16)
    W[0, 0] = 1.0
    x = torch.zeros((4, d), device="cuda", dtype=torch.bfloat16)
    x[:, 0] = torch.tensor([8.0, 16.0, 24.0, 3e4], device="cuda")
    labels = torch.zeros(4, dtype=torch.int64, device="cuda")
    loss, _ = ctx.class_loss(x, W, labels)
    ctx.sync_check()
    want = torch.log1p((classes - 1) * torch.exp(-x[:, 0].double()))
    # log of 1 + s in fp32: the sum is rounded to u of 1
    assert ((loss.double() - want).abs() <= 8 * U + want * 2.0 ** -18).all()


def test_same_bits_every_time_and_each_gradient_alone(ctx):
    x, W, labels, g_loss = problem(700, 200, 900, 9, 0.8)
    loss, lse = ctx.class_loss(x, W, labels)
    both = ctx.class_loss_backward(x, W, labels, lse, g_loss)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip((loss, lse), ctx.class_loss(x, W, labels)))
        assert all(torch.equal(a, b) for a, b in zip(both, ctx.class_loss_backward(x, W, labels, lse, g_loss)))
    assert torch.equal(ctx.class_loss_backward(x, W, labels, lse, g_loss, want_g_w=False)[0], both[0])
    assert torch.equal(ctx.class_loss_backward(x, W, labels, lse, g_loss, want_g_x=False)[1], both[1])


def test_gradients_against_differences(ctx):
    """g_x and g_w against differences of the 64-bit loss, to G's rounding."""
    x, W, labels, _ = problem(20, 24, 12, 10)
    g_loss = torch.full((20,), 0.05, device="cuda")
    loss, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g_loss)

    def total(x, W):
        z = x @ W.t()
        return 0.05 * (torch.logsumexp(z, 1) - z.gather(1, labels[:, None])[:, 0]).sum()

    h, xd, wd = 1e-5, x.double(), W.double()
    ref = reference(x, W, labels, g_loss)
    for i, j in [(0, 0), (7, 11), (19, 23)]:
        e = torch.zeros_like(xd)
        e[i, j] = h
        assert abs(float((total(xd + e, wd) - total(xd - e, wd)) / (2 * h)) - float(g_x[i, j])) <= float(ref["g_x"][1][i, j]) + 1e-9
    for i, j in [(0, 0), (7, 11), (11, 23)]:
        e = torch.zeros_like(wd)
        e[i, j] = h
        assert abs(float((total(xd, wd + e) - total(xd, wd - e)) / (2 * h)) - float(g_w[i, j])) <= float(ref["g_w"][1][i, j]) + 1e-9


@pytest.mark.parametrize("n,d,classes", [(40000, 64, 5000), (20000, 128, 9000)])
def test_pieces_of_rows_and_classes(ctx, n, d, classes):
    """More rows and classes than one piece of G holds: sums over pieces in fp32."""
    x, W, labels, g_loss = problem(n, d, classes, 11, 0.9)
    loss, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g_loss)
    ctx.sync_check()
    gw = torch.zeros((classes, d), dtype=torch.float64, device="cuda")
    room = torch.zeros_like(gw)
    for a in range(0, n, 4000):
        r = slice(a, a + 4000)
        ref = reference(x[r], W, labels[r], g_loss[r])
        for name, got in (("loss", loss), ("lse", lse), ("g_x", g_x)):
            assert ((got[r].double() - ref[name][0]).abs() <= ref[name][1] + 1e-38).all(), (name, a)
        gw += ref["g_w"][0]
        room += ref["g_w"][1]
    assert ((g_w.double() - gw).abs() <= room * 1.5).all()     # the chain of the whole depth: n / 16 steps, ten times a block's


def test_many_rows_few_classes(ctx):
    n, d, classes = 600_000, 32, 47
    x, W, labels, g_loss = problem(n, d, classes, 12, 0.08)
    loss, lse = ctx.class_loss(x, W, labels)
    g_x, g_w = ctx.class_loss_backward(x, W, labels, lse, g_loss)
    ctx.sync_check()
    ref = reference(x, W, labels, g_loss)
    for name, got in (("loss", loss), ("lse", lse), ("g_x", g_x), ("g_w", g_w)):
        assert ((got.double() - ref[name][0]).abs() <= ref[name][1] + 1e-38).all(), name


def test_captured_and_replayed():
    from paper_2210_13149_b200 import binding as B
    stream = torch.cuda.Stream()
    x, W, labels, g_loss = problem(300, 64, 500, 13, 0.7)
    x2, _, labels2, _ = problem(300, 64, 500, 14, 0.3)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = B.BiGCN(0)
        _, lse = c.class_loss(x, W, labels)
        c.class_loss_backward(x, W, labels, lse, g_loss)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            loss, lse = c.class_loss(x, W, labels)
            out = (loss, lse) + c.class_loss_backward(x, W, labels, lse, g_loss)
        x.copy_(x2)
        labels.copy_(labels2)
        c.class_loss(*problem(4000, 64, 800, 15)[:3])
        graph.replay()
        stream.synchronize()
        loss, lse = c.class_loss(x, W, labels)
        want = (loss, lse) + c.class_loss_backward(x, W, labels, lse, g_loss)
        c.sync_check()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_no_rows(ctx):
    x, W, labels, g_loss = problem(4, 32, 10, 16)
    loss, lse = ctx.class_loss(x[:0], W, labels[:0])
    g_x, g_w = ctx.class_loss_backward(x[:0], W, labels[:0], lse, g_loss[:0])
    ctx.sync_check()
    assert loss.numel() == 0 and g_x.shape == (0, 32) and (g_w == 0).all()


def test_strided_outputs_keep_what_lies_between_their_rows(ctx):
    from paper_2210_13149_b200 import binding as B
    x, W, labels, g_loss = problem(90, 40, 30, 17, 0.6)
    loss, lse = ctx.class_loss(x, W, labels)
    want = ctx.class_loss_backward(x, W, labels, lse, g_loss)
    for ld in (43, 48):
        g_x, g_w = torch.full((91, ld), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((31, ld), 7.0, device="cuda", dtype=torch.bfloat16)
        ctx._check(ctx.lib.bigcn_class_loss_backward(ctx.h, B._ptr(x), B._ptr(W), 1, 90, 40, 30, 40, 40, B._ptr(labels), B._ptr(lse), B._ptr(g_loss),
                                                     B._ptr(g_x), ld, B._ptr(g_w), ld))
        ctx.sync_check()
        assert torch.equal(g_x[:90, :40], want[0]) and torch.equal(g_w[:30, :40], want[1])
        assert (g_x[:, 40:] == 7).all() and (g_x[90] == 7).all() and (g_w[:, 40:] == 7).all() and (g_w[30] == 7).all()


def test_refusals(ctx):
    from paper_2210_13149_b200 import binding as B
    x, W, labels, g_loss = problem(8, 32, 10, 18)
    loss, lse = ctx.class_loss(x, W, labels)
    for bad in (lambda: ctx.class_loss(x.float(), W, labels), lambda: ctx.class_loss(x, W.float(), labels), lambda: ctx.class_loss(x, W[:, :16], labels),
                lambda: ctx.class_loss(x, W, labels.int()), lambda: ctx.class_loss(x, W, labels[:7]), lambda: ctx.class_loss(x.t(), W, labels),
                lambda: ctx.class_loss(x.cpu(), W, labels), lambda: ctx.class_loss_backward(x, W, labels, lse[:7], g_loss),
                lambda: ctx.class_loss_backward(x, W, labels, lse, g_loss.double())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.BigcnError):
        ctx.class_loss_backward(x, W, labels, lse, g_loss, want_g_x=False, want_g_w=False)

    def call(**kw):
        a = dict(x=B._ptr(x), w=B._ptr(W), t=1, n=8, d=32, c=10, ldx=32, ldw=32, y=B._ptr(labels), loss=B._ptr(loss), lse=B._ptr(lse))
        a.update(kw)
        return ctx.lib.bigcn_class_loss(ctx.h, *[a[k] for k in ("x", "w", "t", "n", "d", "c", "ldx", "ldw", "y", "loss", "lse")])

    assert call() == 0
    assert call(t=0) == 7 and call(t=3) == 7 and call(d=16385, ldx=16385, ldw=16385) == 7
    assert call(n=-1) == 2 and call(d=0) == 2 and call(c=0) == 2 and call(ldx=31) == 2 and call(ldw=31) == 2
    assert call(x=None) == 1 and call(w=None) == 1 and call(y=None) == 1 and call(loss=None) == 1 and call(lse=None) == 1
    assert call(x=x.data_ptr() + 1) == 3 and call(y=labels.data_ptr() + 4) == 3
    assert ctx.lib.bigcn_class_loss_workspace_bytes(-1, 8, 8, 0) == 0 and ctx.lib.bigcn_class_loss_workspace_bytes(8, 8, 0, 1) == 0
    c = B.BiGCN(0)
    assert c.lib.bigcn_class_loss(c.h, B._ptr(x), B._ptr(W), 1, 8, 32, 10, 32, 32, B._ptr(labels), B._ptr(loss), B._ptr(lse)) == 5
    c.close()
    ctx.sync_check()

"""Layer norm of rows and its gradients, against the formulas in 64 bits.

Tolerances, u = 2^-24: a row is summed by chains of at most 16 values and trees of at most 10 steps, so its mean is off by 26 u times
the mean magnitude, and sums of products by 28 u of theirs; what follows is a handful of roundings.  32 u and 64 u cover them.  An
output of a type with machine epsilon e adds e / 2 of its value, and below fp16's normal range half a step, 2^-25."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    yield c
    c.close()


def rows(n, d, dtype, seed, pad=0, shift=0):
    """Rows of spreads and means of their own; `pad`: of a wider matrix, `shift`: from an odd element on."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, d + pad + shift), device="cuda", generator=gen)
    x = (x + torch.randn((n, 1), device="cuda", generator=gen)) * (torch.rand((n, 1), device="cuda", generator=gen) * 1.5 + 0.25)
    return x.to(dtype)[:, shift:shift + d]


def forward_reference(x, gain, offset, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = ((x - mean[:, None]).square().mean(1) + eps).rsqrt()
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if gain is None else gain.double()
    o = torch.zeros_like(g) if offset is None else offset.double()
    return xhat * g + o, mean, rstd, g.abs() * (32 * rstd[:, None] * x.abs().mean(1)[:, None] + 64 * xhat.abs()) + 4 * o.abs()


def half_step(y, dtype):
    return y.abs() * (torch.finfo(dtype).eps / 2) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def check_forward(ctx, x, gain, offset, eps, out):
    y, mean, rstd = ctx.layer_norm(x, gain, offset, eps=eps, out_dtype=out)
    ctx.sync_check()
    want, m, r, room = forward_reference(x, gain, offset, eps)
    assert y.dtype == out and y.shape == x.shape
    # a value a hair above a rounding border may round the other way: the fp32 error moves the rounded value by as much again
    assert ((y.double() - want).abs() <= half_step(want, out) + 2 * U * room).all()
    assert ((mean.double() - m).abs() <= 32 * U * x.double().abs().mean(1)).all()
    slack = 64 * U * r + 32 * U * r * r * x.double().abs().mean(1)          # the mean's error moves the squares about it, too
    assert ((rstd.double() - r).abs() <= slack).all()


def backward_reference(g, x, mean, rstd, gain):
    g, r = g.double(), rstd.double()[:, None]
    xhat = (x.double() - mean.double()[:, None]) * r
    gg = g if gain is None else g * gain.double()
    a, b = gg.mean(1, keepdim=True), (gg * xhat).mean(1, keepdim=True)
    room = r * (gg.abs() + gg.abs().mean(1, keepdim=True) + xhat.abs() * (gg * xhat).abs().mean(1, keepdim=True))
    return r * (gg - a - xhat * b), (g * xhat).sum(0), g.sum(0), room, (g * xhat).abs().sum(0), g.abs().sum(0)


def check_backward(ctx, g, x, gain, out):
    n, d = x.shape
    _, mean, rstd = ctx.layer_norm(x, gain)
    gx, gg, go = ctx.layer_norm_backward(g, x, mean, rstd, gain, out_dtype=out)
    ctx.sync_check()
    want, wg, wo, room, sg, so = backward_reference(g, x, mean, rstd, gain)
    assert gx.dtype == out
    assert ((gx.double() - want).abs() <= half_step(want, out) + 64 * 2 * U * room).all()
    # a lane adds at most its share of the rows (four rows a warp share it at least), then 8 warps and the rest in 64 bits
    chain = n / 2 + 16 if n < 600 else n / 296 + 16
    assert ((gg.double() - wg).abs() <= (chain + 4) * U * sg + U * wg.abs()).all()
    assert ((go.double() - wo).abs() <= chain * U * so + U * wo.abs()).all()
    again = ctx.layer_norm_backward(g, x, mean, rstd, gain, out_dtype=out)
    assert all(torch.equal(p, q) for p, q in zip((gx, gg, go), again))      # fixed parts, fixed order


@pytest.mark.parametrize("n,d", [(1, 1), (3, 2), (5, 3), (301, 7), (9, 16), (300, 17), (2708, 64), (33, 100), (7, 128), (129, 129), (65, 256),
                                 (64, 500), (31, 602), (17, 1000), (9, 1433), (5, 2049), (4, 4097), (3, 8191), (2, 16384)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_every_length(ctx, n, d, dtype):
    gain = torch.rand(d, device="cuda") + 0.5
    offset = torch.randn(d, device="cuda")
    for out in TYPES:
        check_forward(ctx, rows(n, d, dtype, 1), gain, offset, 1e-5, out)
    check_forward(ctx, rows(n, d, dtype, 2), None, None, 1e-3, dtype)


@pytest.mark.parametrize("n,d", [(1, 2), (5, 3), (301, 7), (9, 16), (300, 17), (2708, 64), (33, 100), (7, 128), (129, 129), (65, 256), (64, 500),
                                 (31, 602), (17, 1000), (9, 1433), (5, 2049), (4, 4097), (3, 8191), (2, 16384), (5000, 48)])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_every_length(ctx, n, d, dtype):
    gain = torch.rand(d, device="cuda") + 0.5
    for gtype in TYPES:
        check_backward(ctx, rows(n, d, gtype, 3) * 0.02, rows(n, d, dtype, 4), gain, torch.float32)
    check_backward(ctx, rows(n, d, dtype, 5) * 0.02, rows(n, d, dtype, 6), None, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (0, 1), (3, 4)])
def test_rows_of_a_wider_matrix(ctx, dtype, pad, shift):
    gain, offset = torch.rand(100, device="cuda") + 0.5, torch.randn(100, device="cuda")
    x = rows(77, 100, dtype, 7, pad, shift)
    check_forward(ctx, x, gain, offset, 1e-5, dtype)
    check_backward(ctx, rows(77, 100, torch.bfloat16, 8, shift, pad), x, gain, dtype)


def test_a_strided_output_keeps_what_lies_between_its_rows(ctx):
    from paper_2210_13149_b200 import binding as B
    x = rows(50, 60, torch.float32, 9)
    y = torch.full((50, 70), 7.0, device="cuda", dtype=torch.bfloat16)
    mean, rstd = torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    ctx._check(ctx.lib.bigcn_layer_norm(ctx.h, B._ptr(x), 0, 50, 60, 60, None, None, 1e-5, B._ptr(y), 1, 70, B._ptr(mean), B._ptr(rstd)))
    ctx.sync_check()
    assert torch.equal(y[:, 60:], torch.full_like(y[:, 60:], 7.0))
    assert torch.equal(y[:, :60], ctx.layer_norm(x, out_dtype=torch.bfloat16)[0])


def test_long_column_sums(ctx):
    """As many rows as the largest graph has, of few columns: the sums over the nodes stay near fp32's own rounding."""
    n, d = 2_449_029, 16
    x, g = rows(n, d, torch.float32, 10), rows(n, d, torch.float32, 11) * 0.02 + 0.001
    _, mean, rstd = ctx.layer_norm(x)
    _, gg, go = ctx.layer_norm_backward(g, x, mean, rstd)
    _, wg, wo, _, _, _ = backward_reference(g, x, mean, rstd, None)
    # 64 rows at a time per block, 296 blocks: 130 rows to a lane's chain, whose roundings are independent
    assert float((gg.double() - wg).norm() / wg.norm()) < 1e-6 and float((go.double() - wo).norm() / wo.norm()) < 1e-6


def test_constant_rows_and_a_row_that_is_not_finite(ctx):
    x = rows(40, 64, torch.float32, 12)
    x[3] = 2.5
    x[7] = 0.0
    want, *_ = ctx.layer_norm(x)
    bad = x.clone()
    bad[11, 5], bad[12, 0], bad[13, 63] = float("nan"), float("inf"), float("-inf")
    got, mean, rstd = ctx.layer_norm(bad)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[11:14] = False
    assert torch.equal(got[keep], want[keep]) and torch.isnan(got[11:14]).all()
    assert torch.isfinite(want).all() and (want[7] == 0).all() and want[3].abs().max() < 1e-3


def test_no_rows(ctx):
    x = torch.empty((0, 32), device="cuda")
    y, mean, rstd = ctx.layer_norm(x)
    assert y.shape == (0, 32) and mean.numel() == 0
    gx, gg, go = ctx.layer_norm_backward(x, x, mean, rstd)
    ctx.sync_check()
    assert gx.shape == (0, 32) and (gg == 0).all() and (go == 0).all()


def test_gradients_against_differences(ctx):
    """The gradients as differences of the 64-bit forward pass: truncation h^2 |y'''| and roundings 2^-53 / h are far below 1e-6."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    x, g = (torch.randn((6, 24), device="cuda", generator=gen) for _ in range(2))
    gain, offset = torch.rand(24, device="cuda", generator=gen) + 0.5, torch.randn(24, device="cuda", generator=gen)
    _, mean, rstd = ctx.layer_norm(x, gain, offset)
    gx, gg, go = ctx.layer_norm_backward(g, x, mean, rstd, gain)
    h = 1e-5

    def loss(x, gain, offset):
        return (forward_reference(x, gain, offset, 1e-5)[0] * g.double()).sum()

    for i, j in [(0, 0), (2, 7), (5, 23)]:
        e = torch.zeros_like(x, dtype=torch.float64)
        e[i, j] = h
        assert abs(float((loss(x.double() + e, gain, offset) - loss(x.double() - e, gain, offset)) / (2 * h)) - float(gx[i, j])) < 2e-5
    for j in (0, 11):
        e = torch.zeros(24, dtype=torch.float64, device="cuda")
        e[j] = h
        assert abs(float((loss(x, gain.double() + e, offset) - loss(x, gain.double() - e, offset)) / (2 * h)) - float(gg[j])) < 2e-5
        assert abs(float((loss(x, gain, offset.double() + e) - loss(x, gain, offset.double() - e)) / (2 * h)) - float(go[j])) < 2e-5


def test_captured_and_replayed(ctx):
    from paper_2210_13149_b200 import binding as B
    stream = torch.cuda.Stream()
    x, g = rows(1000, 96, torch.float32, 14), rows(1000, 96, torch.bfloat16, 15)
    with torch.cuda.stream(stream):
        c = B.BiGCN(0)
        c.layer_norm_backward(g, x, *c.layer_norm(x)[1:])          # the workspace exists before the capture
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y, mean, rstd = c.layer_norm(x)
            out = c.layer_norm_backward(g, x, mean, rstd)
        x2 = rows(1000, 96, torch.float32, 16)
        x.copy_(x2)
        big = rows(3, 16000, torch.float32, 17)
        c.layer_norm_backward(big, big, *c.layer_norm(big)[1:])    # outgrows the workspace that the graph refers to
        graph.replay()
    stream.synchronize()
    want = ctx.layer_norm_backward(g, x2, *ctx.layer_norm(x2)[1:])
    ctx.sync_check()
    assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_refusals(ctx):
    from paper_2210_13149_b200 import binding as B
    x = rows(8, 32, torch.float32, 18)
    mean = torch.empty(8, device="cuda")
    for bad in (x.double(), x.t(), x.cpu(), x[0], x.to(torch.int8)):
        with pytest.raises(ValueError):
            ctx.layer_norm(bad)
    for kw in ({"gain": mean}, {"offset": torch.empty(32, device="cuda", dtype=torch.bfloat16)}, {"out_dtype": torch.int8}):
        with pytest.raises(ValueError):
            ctx.layer_norm(x, **kw)
    with pytest.raises(ValueError):
        ctx.layer_norm_backward(x[:7], x, mean, mean)
    with pytest.raises(ValueError):
        ctx.layer_norm_backward(x, x, mean[:7], mean)
    with pytest.raises(B.BigcnError):
        ctx.layer_norm(x, eps=-1.0)
    with pytest.raises(B.BigcnError) as e:
        ctx.layer_norm(torch.zeros((2, 16385), device="cuda"))
    assert e.value.status == 7

    def call(**kw):
        a = dict(x=B._ptr(x), xt=0, n=8, d=32, ldx=32, y=B._ptr(x), yt=0, ldy=32, mean=B._ptr(mean), rstd=B._ptr(mean), eps=1e-5)
        a.update(kw)
        return ctx.lib.bigcn_layer_norm(ctx.h, a["x"], a["xt"], a["n"], a["d"], a["ldx"], None, None, a["eps"], a["y"], a["yt"], a["ldy"], a["mean"], a["rstd"])

    assert call(x=None) == 1 and call(y=None) == 1 and call(mean=None) == 1 and call(rstd=None) == 1
    assert call(xt=3) == 7 and call(yt=9) == 7 and call(n=-1) == 2 and call(d=0) == 2 and call(ldx=31) == 2 and call(ldy=31) == 2
    assert call(eps=float("nan")) == 2 and call(n=1 << 31) == 2
    assert call(x=x.data_ptr() + 2) == 3


def test_workspace_is_asked_for(ctx):
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    x = rows(8, 32, torch.float32, 19)
    m, out = torch.ones(8, device="cuda"), torch.empty(32, device="cuda")
    gx = torch.empty_like(x)

    def call(gain):
        return c.lib.bigcn_layer_norm_backward(c.h, B._ptr(x), 0, 32, B._ptr(x), 0, 32, 8, 32, None, B._ptr(m), B._ptr(m), B._ptr(gx), 0, 32, gain, None)

    assert call(B._ptr(out)) == 5 and call(None) == 0
    c.sync_check()
    c.close()

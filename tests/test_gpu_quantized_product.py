"""Rows in 8-bit integers and their product with 8-bit class rows: the integers exactly, the product to its roundings.

An output is an exact integer sum rounded to fp32 and two fp32 products, 3 roundings of 2^-24 each, then one to the output's type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ctx():
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    yield c
    c.close()


def rows(n, d, dtype, seed, pad=0, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, d + pad + shift), device="cuda", generator=gen) * (torch.rand((n, 1), device="cuda", generator=gen) * 3 + 0.1)
    return x.to(dtype)[:, shift:shift + d]


def reference_rows(x):
    """The definition, decided by comparisons that 64 bits hold exactly: 127 x against (2 k + 1) top / 2."""
    x = x.double()
    top = x.abs().max(1, keepdim=True).values
    k = torch.floor(127 * x / torch.where(top > 0, top, torch.ones_like(top)))
    beyond = 2 * 127 * x - (2 * k + 1) * top
    q = torch.where((beyond > 0) | ((beyond == 0) & (k.remainder(2) == 1)), k + 1, k)
    return torch.where(top > 0, q, torch.zeros_like(q)), (top / 127).float()[:, 0]


def check_rows(ctx, x):
    q, s = ctx.quantize_rows(x)
    ctx.sync_check()
    want_q, want_s = reference_rows(x)
    d = x.shape[1]
    assert q.shape[1] % 16 == 0 and (q[:, d:] == 0).all()
    assert torch.equal(q[:, :d].double(), want_q) and torch.equal(s, want_s)
    return q, s


LENGTHS = [1, 2, 3, 7, 16, 17, 31, 64, 100, 129, 256, 500, 602, 1000, 1433, 2048, 2049, 4100, 8192, 8193, 16384]


@pytest.mark.parametrize("d", LENGTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_every_length(ctx, d, dtype):
    check_rows(ctx, rows(37 if d < 4000 else 3, d, dtype, d))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (0, 1), (3, 4)])
def test_rows_of_a_wider_matrix(ctx, dtype, pad, shift):
    check_rows(ctx, rows(50, 100, dtype, 1, pad, shift))


def test_halfway_goes_to_the_even_integer(ctx):
    k = torch.arange(-126, 126, device="cuda").float()
    for scale in (1.0, 2.0 ** -30, 2.0 ** 40, 2.0 ** -140, 3.0, 0.7):
        x = torch.cat([k + 0.5, torch.tensor([127.0], device="cuda")])[None, :] * scale
        check_rows(ctx, x)
        for away in (float("inf"), float("-inf")):          # the next fp32 values beside the border
            y = torch.nextafter(x, torch.full_like(x, away))
            y[:, -1] = x[:, -1]
            check_rows(ctx, y)
    q, _ = check_rows(ctx, torch.cat([k + 0.5, torch.tensor([127.0], device="cuda")])[None, :].to(torch.bfloat16))
    assert (q[0, :252] % 2 == 0).all()


def test_rows_of_many_values_near_borders(ctx):
    """Quotients spread over all of (0, 127) with tops of 24 bits: some thousands lie within fp32's rounding of a border."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    top = torch.rand((64, 1), device="cuda", generator=gen) + 1
    k = torch.randint(-127, 127, (64, 8191), device="cuda", generator=gen).double() + 0.5
    x = (k * top.double() / 127).float()
    check_rows(ctx, torch.cat([x, top], 1))


def test_rows_without_values_or_with_values_that_are_not_finite(ctx):
    x = rows(12, 70, torch.float32, 2)
    x[1] = 0.0
    x[2] = -0.0
    x[3, 5], x[4, 0], x[5, 69] = float("nan"), float("inf"), float("-inf")
    x[6] = 2.0 ** -149
    x[7] = 3e38
    q, s = ctx.quantize_rows(x)
    keep = [0, 1, 2, 6, 7, 8, 9, 10, 11]
    want_q, want_s = reference_rows(x[keep])
    assert torch.equal(q[keep, :70].double(), want_q) and torch.equal(s[keep], want_s)
    assert (q[1:6] == 0).all() and (s[1:3] == 0).all() and torch.isnan(s[3:6]).all()
    q_w, s_w = ctx.quantize_rows(rows(9, 70, torch.float32, 3))
    out = ctx.quantized_product(x, q_w, s_w)
    ctx.sync_check()
    assert torch.isnan(out[3:6]).all() and (out[1:3] == 0).all()
    # a row of 3e38 overflows where its product does, and nowhere else
    want = (q[keep].double() @ q_w.double().t()) * s[keep].double()[:, None] * s_w.double()
    fits = want.abs() < 3.4028e38
    assert torch.isinf(out[keep][~fits]).all() and ((out[keep].double() - want)[fits].abs() <= want[fits].abs() * 3.01 * 2.0 ** -24 + 2.0 ** -140).all()


def check_product(ctx, x, w, out):
    q_w, s_w = ctx.quantize_rows(w)
    got = ctx.quantized_product(x, q_w, s_w, out_dtype=out)
    q_x, s_x = ctx.quantize_rows(x)
    again = ctx.quantized_product(q_x, q_w, s_w, s_x=s_x, out_dtype=out)
    ctx.sync_check()
    assert got.dtype == out and got.shape == (x.shape[0], w.shape[0])
    want = (q_x.double() @ q_w.double().t()) * s_x.double()[:, None] * s_w.double()
    tiny = 2.0 ** -25 if out == torch.float16 else 2.0 ** -140
    allow = want.abs() * (3.01 * 2.0 ** -24 + (torch.finfo(out).eps / 2 if out != torch.float32 else 0)) + tiny
    assert ((got.double() - want).abs() <= allow).all()
    assert torch.equal(got, again)


@pytest.mark.parametrize("n,d,m", [(1, 1, 1), (1, 64, 7), (1, 1024, 1000), (1, 602, 30011), (2, 100, 47), (3, 17, 65), (4, 4096, 333), (7, 31, 129),
                                   (8, 256, 40), (9, 500, 7), (16, 128, 256), (23, 602, 1001), (33, 100, 64), (127, 129, 200), (128, 256, 256), (129, 257, 257),
                                   (300, 1433, 70), (1000, 64, 47), (2708, 64, 7), (513, 2049, 513), (40, 16384, 20)])
@pytest.mark.parametrize("dtype", TYPES)
def test_products(ctx, n, d, m, dtype):
    x, w = rows(n, d, dtype, n), rows(m, d, torch.float32, m + 1)
    for out in TYPES:
        check_product(ctx, x, w, out)


@pytest.mark.parametrize("pad,shift", [(8, 0), (5, 0), (0, 1)])
def test_products_of_rows_of_a_wider_matrix(ctx, pad, shift):
    for n in (1, 6, 200):
        check_product(ctx, rows(n, 100, torch.bfloat16, 4, pad, shift), rows(90, 100, torch.float16, 5, pad, shift), torch.float32)


def test_largest_sums_are_exact(ctx):
    x = torch.ones((3, 16384), device="cuda")
    w = torch.ones((5, 16384), device="cuda")
    w[1] = -1
    q_w, s_w = ctx.quantize_rows(w)
    q_x, s_x = ctx.quantize_rows(x)
    assert (q_x == 127).all()
    out = ctx.quantized_product(q_x, q_w, torch.ones_like(s_w), s_x=torch.ones_like(s_x))
    ctx.sync_check()
    want = torch.tensor([127.0 * 127.0 * 16384], device="cuda") * torch.tensor([1.0, -1, 1, 1, 1], device="cuda")
    assert torch.equal(out, want.expand(3, 5))


def test_a_strided_output_keeps_what_lies_between_its_rows(ctx):
    from paper_2210_13149_b200 import binding as B
    q_w, s_w = ctx.quantize_rows(rows(50, 64, torch.float32, 6))
    for n in (1, 5, 140):
        q_x, s_x = ctx.quantize_rows(rows(n, 64, torch.float32, 7))
        out = torch.full((n + 1, 61), 7.0, device="cuda")
        ctx._check(ctx.lib.bigcn_quantized_product(ctx.h, B._ptr(q_x), 3, B._ptr(s_x), n, 64, 64, B._ptr(q_w), 64, B._ptr(s_w), 50, B._ptr(out), 0, 61))
        ctx.sync_check()
        assert (out[:, 50:] == 7).all() and (out[n] == 7).all()
        assert torch.equal(out[:n, :50], ctx.quantized_product(q_x, q_w, s_w, s_x=s_x))


def test_offsets_past_32_bits(ctx):
    """An output of more than 2^32 bytes (and more than 2^31 elements)."""
    n, m = 70_000, 32_768
    x, w = rows(n, 16, torch.bfloat16, 8), rows(m, 16, torch.float32, 9)
    q_w, s_w = ctx.quantize_rows(w)
    q_x, s_x = ctx.quantize_rows(x)
    out = ctx.quantized_product(x, q_w, s_w, out_dtype=torch.bfloat16)
    ctx.sync_check()
    for r in (slice(0, 64), slice(n - 64, n)):
        want = (q_x[r].double() @ q_w.double().t()) * s_x[r].double()[:, None] * s_w.double()
        assert ((out[r].double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -22)).all()


def test_captured_and_replayed():
    from paper_2210_13149_b200 import binding as B
    stream = torch.cuda.Stream()
    x, w = rows(5, 200, torch.float32, 10), rows(300, 200, torch.float32, 11)
    with torch.cuda.stream(stream):
        c = B.BiGCN(0)
        q_w, s_w = c.quantize_rows(w)
        c.quantized_product(x, q_w, s_w)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = c.quantized_product(x, q_w, s_w)
        x.copy_(rows(5, 200, torch.float32, 12))
        c.quantized_product(rows(4000, 1000, torch.float32, 13), *c.quantize_rows(rows(30, 1000, torch.float32, 14)))   # a larger workspace
        graph.replay()
        stream.synchronize()
        assert torch.equal(out, c.quantized_product(x, q_w, s_w))
        c.sync_check()


def test_no_rows(ctx):
    q_w, s_w = ctx.quantize_rows(rows(10, 40, torch.float32, 15))
    assert ctx.quantized_product(torch.empty((0, 40), device="cuda"), q_w, s_w).shape == (0, 10)
    q, s = ctx.quantize_rows(torch.empty((0, 40), device="cuda"))
    assert q.shape == (0, 48) and s.numel() == 0


def test_refusals(ctx):
    from paper_2210_13149_b200 import binding as B
    x, w = rows(4, 40, torch.float32, 16), rows(10, 40, torch.float32, 17)
    q_w, s_w = ctx.quantize_rows(w)
    q_x, s_x = ctx.quantize_rows(x)
    for bad in (lambda: ctx.quantize_rows(x.double()), lambda: ctx.quantize_rows(x.t()), lambda: ctx.quantized_product(x, q_w, s_w[:9]),
                lambda: ctx.quantized_product(x, q_w, s_w, s_x=s_x), lambda: ctx.quantized_product(q_x, q_w, s_w), lambda: ctx.quantized_product(x[:, :20], q_w, s_w),
                lambda: ctx.quantized_product(x, q_w.float(), s_w), lambda: ctx.quantized_product(x, q_w, s_w, out_dtype=torch.int8),
                lambda: ctx.quantized_product(x.cpu(), q_w, s_w)):
        with pytest.raises(ValueError):
            bad()
    out = torch.empty((4, 10), device="cuda")

    def call(**kw):
        a = dict(x=B._ptr(q_x), t=3, s=B._ptr(s_x), n=4, d=40, ldx=48, qw=B._ptr(q_w), ldqw=48, sw=B._ptr(s_w), m=10, out=B._ptr(out), ot=0, ldo=10)
        a.update(kw)
        return ctx.lib.bigcn_quantized_product(ctx.h, *[a[k] for k in ("x", "t", "s", "n", "d", "ldx", "qw", "ldqw", "sw", "m", "out", "ot", "ldo")])

    assert call() == 0
    assert call(m=0) == 2 and call(n=-1) == 2 and call(d=0) == 2 and call(ldo=9) == 2 and call(ldx=39) == 2
    assert call(ldx=40) == 3 and call(ldqw=40) == 3 and call(qw=q_w.data_ptr() + 8) == 3 and call(out=out.data_ptr() + 2) == 3
    assert call(x=None) == 1 and call(s=None) == 1 and call(qw=None) == 1 and call(sw=None) == 1 and call(out=None) == 1
    assert call(ot=3) == 7 and call(t=4) == 7 and call(d=16385, ldx=16400, ldqw=16400) == 7
    c = B.BiGCN(0)
    assert c.lib.bigcn_quantized_product(c.h, B._ptr(x), 0, None, 4, 40, 40, B._ptr(q_w), 48, B._ptr(s_w), 10, B._ptr(out), 0, 10) == 5
    c.close()
    ctx.sync_check()

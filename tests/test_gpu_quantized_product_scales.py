"""8-bit products whose two scales, multiplied, leave fp32's range though the output is inside it: below it digits are lost that the sum brings back, above it
a sum of zero is no number.

An output is the sum rounded to fp32 and two fp32 products, 3 roundings of 2^-24 each, then one to the output's type; below the type's normal range half of
its smallest step."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    yield c
    c.close()


def integers(n, d, seed):
    """Rows of integers, every other one the negative of the one before in half of its columns: some sums are zero."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.zeros((n, (d + 15) // 16 * 16), dtype=torch.int8, device="cuda")
    q[:, :d] = torch.randint(100, 128, (n, d), device="cuda", generator=gen).to(torch.int8)
    q[0, :d] = 127
    q[n // 2:, 1:d:2] *= -1
    if n > 1:
        q[-1, :d] = torch.where(torch.arange(d, device="cuda") % 2 == 0, 127, -127).to(torch.int8)      # times the first row's 127s: zero where d is even
    return q


def check(ctx, q_x, s_x, q_w, s_w, out, got):
    want = (q_x.double() @ q_w.double().t()) * s_x.double()[:, None] * s_w.double()
    least = 2.0 ** -150 if out == torch.float32 else 2.0 ** -134        # half of the smallest step
    top = torch.finfo(out).max
    fits = want.abs() < top * (1 - 2.0 ** -7)
    beyond = want.abs() > top * (1 + 2.0 ** -7)
    room = want.abs() * (3.01 * 2.0 ** -24 + (torch.finfo(out).eps / 2 if out != torch.float32 else 0)) + 3.01 * least
    assert ((got.double() - want).abs() <= room)[fits].all()
    assert (got[beyond] == torch.where(want[beyond] > 0, float("inf"), float("-inf"))).all()
    assert (got[want == 0] == 0).all()
    return int((want == 0).sum())


# One, a few (classes as rows of the tiles), one tile and pairs of tiles; narrow and wide; results on and off 16-byte boundaries.
SHAPES = [(1, 4096, 500), (3, 1000, 70), (40, 512, 333), (64, 4096, 1000), (100, 4096, 40), (129, 256, 129), (300, 4096, 259), (300, 512, 264)]


@pytest.mark.parametrize("n,d,m", SHAPES)
@pytest.mark.parametrize("low,high", [(-80, -70), (-70, -80), (-100, -49), (-149, -1), (-1, -140), (121, 20), (20, 121), (121, 120), (121, -121), (-121, 121), (0, 0)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_scales_of_integer_rows(ctx, n, d, m, low, high, out):
    q_x, q_w = integers(n, d, n), integers(m, d, m + 1)
    gen = torch.Generator(device="cuda").manual_seed(d)
    s_x = (torch.rand(n, device="cuda", generator=gen).double() + 0.5).mul_(2.0 ** low).float()
    s_w = (torch.rand(m, device="cuda", generator=gen).double() + 0.5).mul_(2.0 ** high).float()
    got = ctx.quantized_product(q_x, q_w, s_w, s_x=s_x, out_dtype=out)
    ctx.sync_check()
    assert check(ctx, q_x, s_x, q_w, s_w, out, got) > 0
    # a scale that is no number still shows in its row and its column alone
    s_x[n // 2], s_w[m // 3] = float("nan"), float("nan")
    again = ctx.quantized_product(q_x, q_w, s_w, s_x=s_x, out_dtype=out)
    ctx.sync_check()
    bad = torch.isnan(s_x)[:, None] | torch.isnan(s_w)
    assert torch.isnan(again[bad]).all() and torch.equal(again[~bad], got[~bad])


@pytest.mark.parametrize("n,d,m", [(1, 4096, 500), (2, 512, 300), (4, 1024, 333), (23, 602, 1001), (300, 512, 40)])
@pytest.mark.parametrize("low,high", [(-73, -77), (-100, -40), (126, 20), (20, 126), (126, -110)])
def test_scales_of_rows_quantised_on_the_way(ctx, n, d, m, low, high):
    """Their integers and scales are quantize_rows()'s, and so is the product."""
    x = (integers(n, d, n)[:, :d].double() * 2.0 ** (low - 7)).float()
    q_w = integers(m, d, m + 1)
    s_w = torch.full((m,), 2.0 ** high, device="cuda")
    q_x, s_x = ctx.quantize_rows(x)
    got = ctx.quantized_product(x, q_w, s_w)
    ctx.sync_check()
    assert check(ctx, q_x, s_x, q_w, s_w, torch.float32, got) > 0
    assert torch.equal(got, ctx.quantized_product(q_x, q_w, s_w, s_x=s_x))

"""The norm's gradients for rows whose mean times rstd is past fp32's range though every value of theirs is inside it: lanes that have no column
take no part in the row's sums.

Tolerances, u = 2^-24, h = g gain: a mean of d terms is summed in chains of at most 16 in a lane, then by halves over the lanes and warps: 40 u of the
terms' mean magnitude covers chains, halves and the factor 1 / d; each of the three terms of a result, with xhat's own two roundings, 6 u of it; then the
output's half step.  The columns' sums: chains of n <= 64 rows, 70 u of the terms' magnitudes."""
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


# Words of a row that are cut (d no multiple of 4 or 8) and lanes without a word, for a part of a warp, a warp, several warps and a whole block; rows on and off
# 16-byte boundaries.
@pytest.mark.parametrize("d,ld", [(3, 4), (10, 12), (23, 23), (23, 24), (100, 104), (100, 101), (500, 512), (500, 500), (515, 520), (1030, 1032), (2050, 2051), (4100, 4104),
                                  (8201, 8208), (8201, 8201)])
@pytest.mark.parametrize("dtype,g_dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_rows_far_from_zero(ctx, d, ld, dtype, g_dtype):
    n, eps = 12, 1e-5
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((n, ld), device="cuda", generator=gen).to(dtype)[:, :d]
    far = torch.tensor([1, 4, 11], device="cuda")
    x[far] = 2.0 ** 120
    x[far[1]] = -2.0 ** 121
    g = torch.randn((n, ld), device="cuda", generator=gen).to(g_dtype)[:, :d]
    gain = torch.rand(d, device="cuda", generator=gen) + 0.5
    mean = x.double().mean(1).float()
    rstd = (1 / (((x.double() - mean.double()[:, None]) ** 2).mean(1) + eps).sqrt()).float()
    assert torch.isinf(mean[far] * rstd[far]).all() and (x[far].float() == mean[far, None]).all()
    g_x, g_gain, g_offset = ctx.layer_norm_backward(g, x, mean, rstd, gain)
    ctx.sync_check()
    r, gd = rstd.double()[:, None], g.double()
    xhat = (x.double() - mean.double()[:, None]) * r
    h = gd * gain.double()
    a, b = h.mean(1, keepdim=True), (h * xhat).mean(1, keepdim=True)
    want = r * (h - a - xhat * b)
    room = r * (40 * U * (h.abs().mean(1, keepdim=True) + xhat.abs() * (h * xhat).abs().mean(1, keepdim=True)) + 6 * U * (h.abs() + a.abs() + (xhat * b).abs()))
    if dtype != torch.float32:
        room = room * (1 + 2.0 ** -8) + want.abs() * torch.finfo(dtype).eps / 2
    assert torch.isfinite(g_x).all()
    assert ((g_x.double() - want).abs() <= room + 1e-37).all()
    assert ((g_gain.double() - (gd * xhat).sum(0)).abs() <= 70 * U * (gd * xhat).abs().sum(0) + 1e-37).all()
    assert ((g_offset.double() - gd.sum(0)).abs() <= 70 * U * gd.abs().sum(0) + 1e-37).all()

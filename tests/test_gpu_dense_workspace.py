"""The dense ends keep to the workspace that their sizes ask for: what lies behind it is left, and an exact one is enough."""
import pytest
import torch

pytestmark = pytest.mark.gpu

GUARD = 8 << 20


@pytest.fixture(scope="module")
def ctx():
    from paper_2210_13149_b200 import binding as B
    c = B.BiGCN(0)
    yield c
    c.close()


def exactly(ctx, nbytes):
    """A workspace of nbytes with a guard behind it, both full of NaN patterns."""
    ws = torch.full((nbytes + GUARD,), 255, dtype=torch.uint8, device="cuda")
    ctx.workspace = ws[:nbytes]
    ctx._check(ctx.lib.bigcn_set_workspace(ctx.h, ws.data_ptr(), nbytes))
    return ws


def left(ctx, ws, nbytes):
    ctx.sync_check()
    ok = bool((ws[nbytes:] == 255).all())
    ctx.workspace = None
    ctx._check(ctx.lib.bigcn_set_workspace(ctx.h, None, 0))
    return ok


# Rows that end in the first half of a pair's tile and in the second, one piece of G last in the workspace or parts behind it, few labels
@pytest.mark.parametrize("n,d,classes,labelled", [(8300, 512, 9000, 1.0), (8300, 512, 9000, 0.3), (8200, 500, 9000, 1.0), (300, 96, 300, 1.0), (130, 64, 20000, 1.0),
                                                  (20000, 64, 16500, 1.0), (129, 40, 40, 1.0), (1, 8, 1, 1.0), (8449, 250, 5000, 0.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_class_loss(ctx, n, d, classes, labelled, dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((n, d), device="cuda", generator=gen).to(dtype)
    W = (torch.randn((classes, d), device="cuda", generator=gen) / d ** 0.5).to(dtype)
    y = torch.randint(0, classes, (n,), device="cuda", generator=gen)
    y[torch.rand(n, device="cuda", generator=gen) >= labelled] = -1
    g = torch.rand(n, device="cuda", generator=gen)
    loss, lse = ctx.class_loss(x, W, y)
    g_x, g_w = ctx.class_loss_backward(x, W, y, lse, g)
    for backward in (0, 1):
        need = int(ctx.lib.bigcn_class_loss_workspace_bytes(n, d, classes, backward))
        ws = exactly(ctx, need)
        if backward:
            again = ctx.class_loss_backward(x, W, y, lse, g)
            assert torch.equal(again[0], g_x) and torch.equal(again[1], g_w)
        else:
            again = ctx.class_loss(x, W, y)
            assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
        assert left(ctx, ws, need)


@pytest.mark.parametrize("n,d,m", [(1, 100, 70), (5, 33, 3000), (64, 1000, 65), (129, 250, 40), (300, 96, 300), (5000, 17, 129)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantized_product(ctx, n, d, m, dtype):
    x = torch.randn((n, d), device="cuda").to(dtype)
    q, s = ctx.quantize_rows(torch.randn((m, d), device="cuda"))
    out = ctx.quantized_product(x, q, s)
    need = int(ctx.lib.bigcn_quantized_product_workspace_bytes(n, d))
    ws = exactly(ctx, need)
    assert torch.equal(ctx.quantized_product(x, q, s), out)
    assert left(ctx, ws, need)


@pytest.mark.parametrize("n,d", [(1, 1), (300, 23), (5000, 500), (3000, 4097), (700, 16384)])
def test_layer_norm_backward(ctx, n, d):
    x, g = torch.randn((n, d), device="cuda"), torch.randn((n, d), device="cuda")
    _, mean, rstd = ctx.layer_norm(x)
    want = ctx.layer_norm_backward(g, x, mean, rstd)
    need = int(ctx.lib.bigcn_layer_norm_workspace_bytes(d))
    ws = exactly(ctx, need)
    assert all(torch.equal(a, b) for a, b in zip(ctx.layer_norm_backward(g, x, mean, rstd), want))
    assert left(ctx, ws, need)


def test_leading_dimensions_that_no_tensor_map_holds_are_refused(ctx):
    """One row has no next one, so any leading dimension could be given for it; the products' maps take none of 2^40 bytes."""
    from paper_2210_13149_b200 import binding as B
    x, W = torch.randn((1, 64), device="cuda").bfloat16(), torch.randn((8, 64), device="cuda").bfloat16()
    y, out = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
    q, s = ctx.quantize_rows(W)
    ctx._scratch(1 << 20)
    before = ctx.launch_count()
    far = 1 << 38
    P = B._ptr
    for status in (ctx.lib.bigcn_class_loss(ctx.h, P(x), P(W), 1, 1, 64, 8, far, 64, P(y), P(out), P(out[1:])),
                   ctx.lib.bigcn_class_loss(ctx.h, P(x), P(W), 1, 1, 64, 1, 64, far, P(y), P(out), P(out[1:])),
                   ctx.lib.bigcn_quantized_product(ctx.h, P(q), 3, P(s), 1, 64, far, P(q), 64, P(s), 8, P(out), 0, 8),
                   ctx.lib.bigcn_quantized_product(ctx.h, P(x), 1, None, 1, 64, 64, P(q), far, P(s), 1, P(out), 0, 1)):
        assert status != 0
        with pytest.raises(B.BigcnError):
            ctx._check(status)
    assert ctx.launch_count() == before
    ctx.sync_check()

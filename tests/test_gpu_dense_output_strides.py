"""Leading dimensions of results keep to the documented bound (below 2^38), as those of inputs do: refused before anything is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_leading_dimensions_of_results():
    from paper_2210_13149_b200 import binding as B
    ctx = B.BiGCN(0)
    P, far = B._ptr, 1 << 38
    x, W = torch.randn((1, 64), device="cuda").bfloat16(), torch.randn((1, 64), device="cuda").bfloat16()
    y, one = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    f, mean, rstd, out = torch.randn((1, 64), device="cuda"), torch.zeros(1, device="cuda"), torch.ones(1, device="cuda"), torch.empty((1, 64), device="cuda")
    g_x, g_w = torch.empty_like(x), torch.empty_like(W)
    q, s = ctx.quantize_rows(W)
    ctx.ensure_workspace(1 << 20)

    def calls(ld):
        yield lambda: ctx.lib.bigcn_class_loss_backward(ctx.h, P(x), P(W), 1, 1, 64, 1, 64, 64, P(y), P(one), P(one), P(g_x), ld, P(g_w), 64)
        yield lambda: ctx.lib.bigcn_class_loss_backward(ctx.h, P(x), P(W), 1, 1, 64, 1, 64, 64, P(y), P(one), P(one), P(g_x), 64, P(g_w), ld)
        yield lambda: ctx.lib.bigcn_class_loss_backward(ctx.h, P(x), P(W), 1, 0, 64, 1, 64, 64, None, None, None, P(g_x), 64, P(g_w), ld)
        yield lambda: ctx.lib.bigcn_quantized_product(ctx.h, P(x), 1, None, 1, 64, 64, P(q), 64, P(s), 1, P(out), 0, ld)
        yield lambda: ctx.lib.bigcn_quantized_product(ctx.h, P(q), 3, P(s), 1, 64, 64, P(q), 64, P(s), 1, P(out), 0, ld)
        yield lambda: ctx.lib.bigcn_layer_norm(ctx.h, P(f), 0, 1, 64, 64, None, None, 1e-5, P(out), 0, ld, P(mean), P(rstd))
        yield lambda: ctx.lib.bigcn_layer_norm_backward(ctx.h, P(f), 0, 64, P(f), 0, 64, 1, 64, None, P(mean), P(rstd), P(out), 0, ld, None, None)

    assert all(call() == 0 for call in calls(64))
    ctx.sync_check()
    before = ctx.launch_count()
    assert [call() for call in calls(far)] == [2] * 7
    assert ctx.launch_count() == before
    ctx.sync_check()
    ctx.close()

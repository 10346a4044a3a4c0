"""Captured calls of binarized layers, and eager dense calls that outgrow the workspace they used: a replay writes its own memory and gives its own result."""
import pytest
import torch

from paper_2210_13149_b200 import synth

pytestmark = pytest.mark.gpu


def setting(stream, n=2000, d_in=64, d_out=48):
    from paper_2210_13149_b200 import binding as B
    ctx = B.BiGCN(0, stream)
    G = ctx.normalize_adjacency(*synth.power_law_graph(n, 8 * n, 1, device="cuda"))
    W = synth.weights([d_in, d_out], 1, "cuda")[0]
    layer = ctx.prepare_layers([W])[0]
    gen = torch.Generator(device="cuda").manual_seed(1)
    X = torch.randn((n, d_in), device="cuda", generator=gen)
    g = torch.randn((n, d_out), device="cuda", generator=gen)
    return ctx, G, layer, W, X, g, gen


def dense(gen):
    x = torch.randn((3000, 64), device="cuda", generator=gen).bfloat16()
    C = torch.randn((4000, 64), device="cuda", generator=gen).bfloat16()
    y = torch.randint(0, 4000, (3000,), device="cuda", generator=gen)
    return x, C, y, torch.rand(3000, device="cuda", generator=gen)


@pytest.mark.parametrize("inside", [False, True])
def test_a_larger_workspace_after_the_capture_and_within_it(inside):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx, G, layer, W, X, g, gen = setting(stream)
        x, C, y, gl = dense(gen)
        bits, beta = ctx.pack_features(X)
        # eager results, from a context of their own
        other = setting(stream)[0]
        want = (other.layer_forward(G, layer, bits, beta)["h"], *other.layer_backward(G, layer, W, bits, beta, g))
        loss, lse = other.class_loss(x, C, y)
        want_dense = (loss, lse, *other.class_loss_backward(x, C, y, lse, gl))
        other.sync_check()

        ctx.layer_forward(G, layer, bits, beta)
        ctx.layer_backward(G, layer, W, bits, beta, g)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        got_dense = None
        with torch.cuda.graph(graph, stream=stream):
            got = (ctx.layer_forward(G, layer, bits, beta)["h"], *ctx.layer_backward(G, layer, W, bits, beta, g))
            if inside:
                a, b = ctx.class_loss(x, C, y)
                got_dense = (a, b, *ctx.class_loss_backward(x, C, y, b, gl))
        before = ctx.workspace
        address, size = before.data_ptr(), before.numel()
        del before
        assert any(w.data_ptr() == address for w in ctx._captured)
        # an eager call that needs more, and tensors over all that the allocator has to give
        ctx.class_loss_backward(*[t.repeat(8, *[1] * (t.dim() - 1)) if t.shape[0] == 3000 else t for t in (x, C, y, lse, gl)])
        assert ctx.workspace.numel() > size
        stream.synchronize()
        fill = [torch.full((max(1, size // 4),), 12345, dtype=torch.int32, device="cuda") for _ in range(8)]
        assert all(f.data_ptr() != address for f in fill)
        for t in got + (got_dense or ()):
            t.fill_(float("nan"))
        graph.replay()
        stream.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert not inside or all(torch.equal(p, q) for p, q in zip(got_dense, want_dense))
        assert all((f == 12345).all() for f in fill)
        ctx.sync_check()

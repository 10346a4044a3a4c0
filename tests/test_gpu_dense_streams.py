"""The dense ends from a stream that is not the context's own: memory of neither side is given away while the other still works with it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def calls(ctx):
    """name -> (inputs, call of them); outputs as tuples."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((500, 96), device="cuda", generator=gen)
    g = torch.randn((500, 96), device="cuda", generator=gen)
    W = torch.randn((70, 96), device="cuda", generator=gen).bfloat16()
    y = torch.randint(0, 70, (500,), device="cuda", generator=gen)
    gain, offset = torch.rand(96, device="cuda", generator=gen), torch.rand(96, device="cuda", generator=gen)
    _, mean, rstd = ctx.layer_norm(x)
    xb, g_loss = x.bfloat16(), torch.rand(500, device="cuda", generator=gen)
    _, lse = ctx.class_loss(xb, W, y)
    q, s = ctx.quantize_rows(W)
    torch.cuda.synchronize()
    return {"norm": ((x, gain, offset), ctx.layer_norm),
            "norm backward": ((g, x, mean, rstd, gain), ctx.layer_norm_backward),
            "loss": ((xb, W, y), ctx.class_loss),
            "loss backward": ((xb, W, y, lse, g_loss), ctx.class_loss_backward),
            "rows": ((x,), ctx.quantize_rows),
            "product": ((xb, q, s), lambda *a: (ctx.quantized_product(*a),))}


@pytest.mark.parametrize("name", ["norm", "norm backward", "loss", "loss backward", "rows", "product"])
def test_memory_between_two_streams(name):
    from paper_2210_13149_b200 import binding as B
    side = torch.cuda.Stream()
    ctx = B.BiGCN(0, side)
    inputs, call = calls(ctx)[name]
    want = call(*inputs)
    ctx.sync_check()
    torch.cuda.synchronize()
    here = torch.cuda.current_stream()
    assert here != side

    # inputs that are dropped, and whose memory another tensor would take, before the context's stream reads them
    copies = [t.clone() for t in inputs]
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    side.wait_stream(here)
    got = call(*copies)
    shapes = [(t.shape, t.dtype) for t in copies]
    del copies
    others = [torch.zeros(shape, dtype=dtype, device="cuda") for shape, dtype in shapes]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del others

    # outputs that are dropped while this stream still reads them
    here.wait_stream(side)
    got = call(*inputs)
    here.wait_stream(side)
    torch.cuda._sleep(20_000_000)
    read = [t.clone() for t in got]
    del got
    with torch.cuda.stream(side):
        others = [torch.zeros_like(t) for t in want]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(read, want))
    ctx.close()


def test_one_row_of_8_bits_that_is_a_part_of_its_row():
    """One row of 100 integers in a row of 112, as two such rows are taken."""
    from paper_2210_13149_b200 import binding as B
    ctx = B.BiGCN(0)
    q_w, s_w = ctx.quantize_rows(torch.randn((30, 100), device="cuda"))
    q, s = ctx.quantize_rows(torch.randn((2, 100), device="cuda"))
    two = ctx.quantized_product(q[:, :100], q_w, s_w, s)
    one = ctx.quantized_product(q[:1, :100], q_w, s_w, s[:1])
    one_class = ctx.quantized_product(q, q_w[:1, :100], s_w[:1], s)
    ctx.sync_check()
    assert torch.equal(one, two[:1]) and torch.equal(one_class, two[:, :1])
    ctx.close()

"""The dense ends in a row with binarized layers, as a training step and as serving use them, and calls beside each other."""
import pytest
import torch

from paper_2210_13149_b200 import synth

pytestmark = pytest.mark.gpu


def network(seed, n=3000, d_in=100, hidden=96, classes=300):
    from paper_2210_13149_b200 import binding as B
    ctx = B.BiGCN(0)
    G = ctx.normalize_adjacency(*synth.power_law_graph(n, 8 * n, seed, device="cuda"))
    W = synth.weights([d_in, hidden], seed, "cuda")[0]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((n, d_in), device="cuda", generator=gen)
    C = torch.randn((classes, hidden), device="cuda", generator=gen) / hidden ** 0.5
    labels = torch.randint(0, classes, (n,), device="cuda", generator=gen)
    labels[torch.rand(n, device="cuda", generator=gen) < 0.6] = -1
    gain, offset = torch.rand(hidden, device="cuda", generator=gen) + 0.5, torch.randn(hidden, device="cuda", generator=gen) * 0.1
    return ctx, G, W, X, C, labels, gain, offset


def test_training_step():
    """Binarized layer, norm, loss and back: every gradient against 64 bits from the layer's own output.

    Between that and here lie three roundings to bf16 (the normed rows, G, the gradient of the normed rows), 2^-8 of a value each at most, which
    the norm's gradient (a projection, times the rows' scale) does not enlarge relative to its result's 2-norm by more than the gradients' sums
    lose: 4 * 2^-8 covers the three in the 2-norm."""
    ctx, G, W, X, C, labels, gain, offset = network(3)
    layer = ctx.prepare_layers([W])[0]
    bits, beta = ctx.pack_features(X)
    H = ctx.layer_forward(G, layer, bits, beta)["h"]
    Y, mean, rstd = ctx.layer_norm(H, gain, offset, out_dtype=torch.bfloat16)
    Cb = C.bfloat16()
    loss, lse = ctx.class_loss(Y, Cb, labels)
    kept = labels >= 0
    g_loss = torch.full_like(loss, 1.0 / int(kept.sum()))
    g_y, g_c = ctx.class_loss_backward(Y, Cb, labels, lse, g_loss)
    g_h, g_gain, g_offset = ctx.layer_norm_backward(g_y, H, mean, rstd, gain)
    _, g_w = ctx.layer_backward(G, layer, W, bits, beta, g_h, want_g_in=False)
    ctx.sync_check()

    leaves = [t.double().requires_grad_() for t in (H, gain, offset, Cb)]
    h, ga, of, c = leaves
    y = (h - h.mean(1, keepdim=True)) * (h.var(1, unbiased=False, keepdim=True) + 1e-5).rsqrt() * ga + of
    total = torch.nn.functional.cross_entropy((y @ c.t())[kept], labels[kept])
    want = torch.autograd.grad(total, leaves)
    assert abs(float(loss.double().sum() / kept.sum()) - float(total.detach())) < 2e-2 * float(total.detach()) * 2.0 ** -4
    for got, ref in zip((g_h, g_gain, g_offset, g_c), want):
        assert float((got.double() - ref).norm() / ref.norm()) < 4 * 2.0 ** -8
    assert (g_h[~kept] == 0).all()
    # the binarized layer's own gradient from the exact one
    _, g_w_exact = ctx.layer_backward(G, layer, W, bits, beta, want[0].float(), want_g_in=False)
    ctx.sync_check()
    assert float((g_w - g_w_exact).double().norm() / g_w_exact.double().norm()) < 4 * 2.0 ** -8
    ctx.close()


@pytest.mark.parametrize("rows", [1, 5, 3000])
def test_serving(rows):
    """The same class matrix served in 8 bits: every logit within half a step of each of its factors."""
    ctx, G, W, X, C, labels, gain, offset = network(4)
    layer = ctx.prepare_layers([W])[0]
    H = ctx.layer_forward(G, layer, *ctx.pack_features(X))["h"][:rows]
    Y, _, _ = ctx.layer_norm(H, gain, offset)
    q, s = ctx.quantize_rows(C)
    got = ctx.quantized_product(Y, q, s)
    ctx.sync_check()
    y, c = Y.double(), C.double()
    ey, ec = y.abs().amax(1) / 254, c.abs().amax(1) / 254          # half a step of either
    room = ey[:, None] * c.abs().sum(1) + ec * y.abs().sum(1)[:, None] + ey[:, None] * ec * c.shape[1]
    assert ((got.double() - y @ c.t()).abs() <= room * (1 + 2.0 ** -20)).all()
    ctx.close()


def test_contexts_beside_each_other():
    """Two contexts on two streams, their calls interleaved, give what each gives alone; a context used while another stream is current
    allocates on its own."""
    from paper_2210_13149_b200 import binding as B
    gen = torch.Generator(device="cuda").manual_seed(5)
    jobs = []
    for n, d, classes in ((700, 128, 3000), (1500, 72, 900)):
        x = torch.randn((n, d), device="cuda", generator=gen)
        W = torch.randn((classes, d), device="cuda", generator=gen) / d ** 0.5
        labels = torch.randint(0, classes, (n,), device="cuda", generator=gen)
        jobs.append((x, W, labels, torch.rand(n, device="cuda", generator=gen)))
    torch.cuda.synchronize()

    def steps(c, x, W, labels, g):
        y, mean, rstd = c.layer_norm(x, out_dtype=torch.bfloat16)
        Wb = W.bfloat16()
        torch.cuda.current_stream().synchronize()
        yield
        loss, lse = c.class_loss(y, Wb, labels)
        yield
        g_y, g_w = c.class_loss_backward(y, Wb, labels, lse, g)
        yield
        g_x, g_gain, g_offset = c.layer_norm_backward(g_y, x, mean, rstd)
        q, s = c.quantize_rows(W)
        yield
        yield loss, lse, g_y, g_w, g_x, g_gain, g_offset, c.quantized_product(x, q, s), c.quantized_product(x[:2], q, s), Wb

    alone = []
    for job in jobs:
        c = B.BiGCN(0)
        alone.append(list(steps(c, *job))[-1])
        c.sync_check()
        c.close()
    streams = [torch.cuda.Stream() for _ in jobs]
    contexts = [B.BiGCN(0, stream=s) for s in streams]          # the default stream stays current
    for _ in range(5):
        running = [steps(c, *job) for c, job in zip(contexts, jobs)]
        for _ in range(4):
            for r in running:
                next(r)
        out = [next(r) for r in running]
        for c in contexts:
            c.sync_check()
        for a, b in zip(alone, out):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
    for c in contexts:
        c.close()


def test_calls_do_not_touch_their_inputs():
    ctx, G, W, X, C, labels, gain, offset = network(6)
    Cb, x = C.bfloat16(), X[:, :96].contiguous()
    inputs = [x, Cb, labels, gain, offset, C]
    before = [t.clone() for t in inputs]
    y, mean, rstd = ctx.layer_norm(x, gain, offset, out_dtype=torch.bfloat16)
    kept = [y.clone(), mean.clone(), rstd.clone()]
    loss, lse = ctx.class_loss(y, Cb, labels)
    g = torch.ones_like(loss)
    g_y, _ = ctx.class_loss_backward(y, Cb, labels, lse, g)
    ctx.layer_norm_backward(g_y, x, mean, rstd, gain)
    q, s = ctx.quantize_rows(C)
    ctx.quantized_product(x, q, s)
    ctx.sync_check()
    assert all(torch.equal(a, b) for a, b in zip(inputs + [y, mean, rstd], before + kept)) and (g == 1).all()
    ctx.close()

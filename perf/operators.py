"""The dense ends of a node classifier on binarized layers, as measurable cases: the norm of a layer's rows, the loss of a
class matrix with its gradients, and the same matrix served in 8-bit integers.

Kinds of case

  norm            ``BiGCN.layer_norm``: every row centred and scaled to unit variance, with a gain and an offset per column
  norm_backward   ``BiGCN.layer_norm_backward``: the gradients of the rows, of the gain and of the offset
  loss            ``BiGCN.class_loss``: softmax cross entropy of rows against a class matrix, the logits never stored
  loss_step       the same, then ``BiGCN.class_loss_backward``: the gradients of the rows and of the class matrix
  head            ``BiGCN.quantized_product``: rows quantised to 8 bits each with a scale of its own, times a class matrix of
                  8-bit rows with scales of their own

With ``own`` the library's calls run; without it the same operators in elementary torch operations.
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _norm(name, kind, n, d, type, out, pad=0):
    return {"name": name, "kind": kind, "n": n, "d": d, "type": type, "out": out, "pad": pad}


def _loss(name, kind, n, d, classes, labelled=1.0, pad=0):
    return {"name": name, "kind": kind, "n": n, "d": d, "classes": classes, "labelled": labelled, "pad": pad}


def _head(name, n, d, classes, type, out, pad=0):
    return {"name": name, "kind": "head", "n": n, "d": d, "classes": classes, "type": type, "out": out, "pad": pad}


def listed():
    return [
        # Hidden rows of a citation graph: the smallest norm, all latency.
        _norm("citation_norm", "norm", 2_708, 64, "fp32", "fp32"),
        # Hidden rows of the co-purchase graph, handed on in bf16 to a class matrix: the largest norm, all bandwidth.
        _norm("products_norm", "norm", 2_449_029, 256, "fp32", "bf16"),
        # Back through the norm of image-graph rows, of 500 columns in bf16, rows of a wider matrix.
        _norm("image_norm_backward", "norm_backward", 89_250, 500, "bf16", "bf16", pad=12),
        # Back through the norm of the paper graph's hidden rows: bf16 gradients come in, fp32 ones go to the binarized layer.
        _norm("papers_norm_backward", "norm_backward", 169_343, 256, "fp32", "fp32"),
        # One training step's loss on a citation graph: seven classes, one node in nineteen labelled.
        _loss("citation_loss_step", "loss_step", 2_708, 64, 7, 0.052),
        # The co-purchase graph's: 47 classes, one node in twelve labelled.
        _loss("products_loss_step", "loss_step", 2_449_029, 256, 47, 0.08),
        # Evaluation against a large set of classes (items, entities): odd sizes throughout.
        _loss("items_loss", "loss", 1_999, 602, 30_011),
        # Training against a large set of classes, the largest case.
        _loss("entities_loss_step", "loss_step", 8_192, 1_024, 65_536),
        # One node served against a large set of classes: the weights are read once, for one row.
        _head("one_node_head", 1, 1_024, 65_536, "bf16", "fp32"),
        # A few nodes, odd sizes.
        _head("few_nodes_head", 23, 602, 30_011, "fp16", "fp16"),
        # All nodes of the paper graph.
        _head("papers_head", 169_343, 256, 40, "fp32", "fp32"),
        # A large batch against a large set of classes.
        _head("batch_head", 16_384, 2_048, 32_768, "bf16", "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """Another case of the same ranges: sizes spread over their logarithm, round and odd, rows dense or of a wider matrix."""
    kind = rng.choice(["norm", "norm_backward", "loss", "loss_step", "head"])
    pad = rng.choice([0, 0, 8, 5])
    if kind in ("norm", "norm_backward"):
        n = _log_int(rng, 1, 2_449_029)
        d = _log_int(rng, 16, min(8_192, 200_000_000 // n))
        if rng.random() < 0.5 and d >= 64:
            d -= d % 64
        case = _norm("", kind, n, d, rng.choice(["fp32", "bf16", "fp16"]), rng.choice(["fp32", "bf16", "fp16"]), pad)
    else:
        d = _log_int(rng, 16, 4_096)
        if rng.random() < 0.5 and d >= 64:
            d -= d % 64
        classes = _log_int(rng, 2, 131_072)
        n = _log_int(rng, 1, max(1, min(300_000, 500_000_000 // max(classes, d), 200_000_000_000 // (classes * d))))
        if kind == "head":
            case = _head("", n, d, classes, rng.choice(["fp32", "bf16", "fp16"]), rng.choice(["fp32", "bf16", "fp16"]), pad)
        else:
            case = _loss("", kind, n, d, classes, rng.choice([1.0, 1.0, 0.5, 0.08]), pad)
    del case["name"]
    return case


_kept = {}


def _context():
    """The library context that a program keeps for its run."""
    if "ctx" not in _kept:
        from paper_2210_13149_b200 import binding
        _kept["ctx"] = binding.BiGCN(0)
    return _kept["ctx"]


def _rows(n, d, pad, dtype, gen, spread=None):
    """Random rows, dense or the first columns of a wider matrix."""
    x = torch.randn((n, d + pad), device="cuda", generator=gen)
    if spread is not None:
        x[:, :d].mul_(spread)
    return x.to(dtype)[:, :d]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed % 1_000_003 + 17)
    kind, n, d, pad = case["kind"], case["n"], case["d"], case["pad"]
    s = {"case": case}
    if own:
        s["ctx"] = _context()
    if kind in ("norm", "norm_backward"):
        # Rows with a spread and a mean of their own, as aggregated activations have: wide at hubs, narrow elsewhere.
        x = torch.randn((n, d + pad), device="cuda", generator=gen)
        x.add_(torch.randn((n, 1), device="cuda", generator=gen)).mul_(torch.rand((n, 1), device="cuda", generator=gen) * 1.5 + 0.25)
        s["x"] = x.to(_TYPES[case["type"]])[:, :d]
        del x
        s["gain"] = torch.rand(d, device="cuda", generator=gen) + 0.5
        s["offset"] = torch.randn(d, device="cuda", generator=gen) * 0.2
        s["eps"] = 1e-5
        if kind == "norm_backward":
            # The gradient comes from the layer behind in bf16, or in the rows' own type.
            s["g_y"] = _rows(n, d, pad, torch.bfloat16 if case["out"] == "bf16" else _TYPES[case["type"]], gen, 0.02)
            # What the forward pass kept.
            s["mean"], s["rstd"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            for a in range(0, n, 262_144):
                b = s["x"][a:a + 262_144].double()
                s["mean"][a:a + 262_144] = b.mean(1)
                s["rstd"][a:a + 262_144] = (b.var(1, unbiased=False) + s["eps"]).rsqrt()
        return s
    classes = case["classes"]
    W = torch.randn((classes, d + (pad if kind != "head" else 0)), device="cuda", generator=gen) / math.sqrt(d)
    if kind == "head":
        s["x"] = _rows(n, d, pad, _TYPES[case["type"]], gen, torch.rand((n, 1), device="cuda", generator=gen) * 3 + 0.1)
        # The class matrix, quantised once: 8-bit rows on 16-byte boundaries, and a scale for each.
        top = W.abs().amax(1)
        s["q_w"] = torch.zeros((classes, (d + 15) // 16 * 16), dtype=torch.int8, device="cuda")
        s["q_w"][:, :d] = (W * (127.0 / top)[:, None]).round().to(torch.int8)
        s["s_w"] = top / 127.0
        return s
    # Rows that lean towards their own class, as in training; nodes without a label carry -1.
    s["W"] = W.to(torch.bfloat16)[:, :d]
    labels = torch.randint(0, classes, (n,), device="cuda", generator=gen)
    x = torch.randn((n, d + pad), device="cuda", generator=gen)
    x[:, :d] += W[labels, :d] * (torch.rand((n, 1), device="cuda", generator=gen) * 8)
    s["x"] = x.to(torch.bfloat16)[:, :d]
    if case["labelled"] < 1:
        labels = torch.where(torch.rand(n, device="cuda", generator=gen) < case["labelled"], labels, torch.full_like(labels, -1))
        labels[n // 2] = n % classes  # one at least
    s["labels"] = labels
    # The loss's own gradient: the mean over the labelled nodes.
    s["g_loss"] = torch.full((n,), 1.0, device="cuda") / (labels >= 0).sum().clamp(min=1)
    return s


def _own(s):
    case, ctx, kind = s["case"], s["ctx"], s["case"]["kind"]
    if kind == "norm":
        return ctx.layer_norm(s["x"], s["gain"], s["offset"], eps=s["eps"], out_dtype=_TYPES[case["out"]])
    if kind == "norm_backward":
        return ctx.layer_norm_backward(s["g_y"], s["x"], s["mean"], s["rstd"], s["gain"], out_dtype=_TYPES[case["out"]])
    if kind == "head":
        return ctx.quantized_product(s["x"], s["q_w"], s["s_w"], out_dtype=_TYPES[case["out"]])
    loss, lse = ctx.class_loss(s["x"], s["W"], s["labels"])
    if kind == "loss":
        return loss, lse
    g_x, g_w = ctx.class_loss_backward(s["x"], s["W"], s["labels"], lse, s["g_loss"])
    return loss, lse, g_x, g_w


def run(s):
    if own:
        return _own(s)
    case, kind, x = s["case"], s["case"]["kind"], s["x"]
    if kind == "norm":
        x = x.float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = (c.square().mean(1) + s["eps"]).rsqrt()
        return (c.mul_(rstd[:, None]).mul_(s["gain"]).add_(s["offset"])).to(_TYPES[case["out"]]), mean, rstd
    if kind == "norm_backward":
        xhat = (x.float() - s["mean"][:, None]).mul_(s["rstd"][:, None])
        g = s["g_y"].float()
        # Sums over the nodes are long: in 64 bits.
        g_offset = g.sum(0, dtype=torch.float64).float()
        g_gain = (g * xhat).sum(0, dtype=torch.float64).float()
        g = g * s["gain"]
        a, b = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
        return ((g - a - xhat * b) * s["rstd"][:, None]).to(_TYPES[case["out"]]), g_gain, g_offset
    if kind == "head":
        # In 64 bits: a value halfway between two integers has to be seen as that.
        xd = x.double()
        top = xd.abs().amax(1)
        q = torch.round(xd * 127 / torch.where(top > 0, top, torch.ones_like(top))[:, None]).float()
        out = q @ s["q_w"][:, :case["d"]].float().t()
        return (out * (top / 127).float()[:, None] * s["s_w"]).to(_TYPES[case["out"]])
    labels, kept = s["labels"], s["labels"] >= 0
    xf, wf = x.float(), s["W"].float()
    z = xf[kept] @ wf.t()
    top = z.amax(1)
    total = (z - top[:, None]).exp_().sum(1)
    y = labels[kept]
    at = z.gather(1, y[:, None])[:, 0]
    loss, lse = torch.zeros(x.shape[0], device=x.device), torch.zeros(x.shape[0], device=x.device)
    loss[kept] = (top - at) + total.log()
    lse[kept] = top + total.log()
    if kind == "loss":
        return loss, lse
    g = z.sub_(lse[kept][:, None]).exp_()
    g[torch.arange(y.numel(), device=y.device), y] -= 1
    g.mul_(s["g_loss"][kept][:, None])
    g_x = torch.zeros_like(xf)
    g_x[kept] = g @ wf
    return loss, lse, g_x.to(torch.bfloat16), (g.t() @ xf[kept]).to(torch.bfloat16)


def work(case):
    """Bytes: every input read once, every result written once.  Operations: two for each multiply-add of the products,
    and a few for each element elsewhere."""
    kind, n, d = case["kind"], case["n"], case["d"]
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if kind == "norm":
        return {"bytes": n * d * (size[case["type"]] + size[case["out"]]) + 8 * (n + d), "flops": 8 * n * d}
    if kind == "norm_backward":
        g = 2 if case["out"] == "bf16" else size[case["type"]]
        return {"bytes": n * d * (size[case["type"]] + g + size[case["out"]]) + 8 * n + 12 * d, "flops": 14 * n * d}
    classes = case["classes"]
    if kind == "head":
        return {"bytes": n * d * size[case["type"]] + classes * (d + 4) + n * classes * size[case["out"]], "flops": 2 * n * d * classes}
    rows = max(1, round(n * case["labelled"]))
    if kind == "loss":
        return {"bytes": 2 * d * (rows + classes) + 16 * n, "flops": 2 * rows * d * classes}
    return {"bytes": 2 * d * (rows + classes) + 2 * d * (n + classes) + 20 * n, "flops": 6 * rows * d * classes}


def exact(case, seed):
    """The definitions, in 64 bits, a block of rows at a time."""
    s = prepare(case, seed)
    kind, n, d, f64 = case["kind"], case["n"], case["d"], torch.float64
    if kind == "norm":
        if n * d > 700_000_000:
            return None
        out, means, scales = [], [], []
        for a in range(0, n, 131_072):
            x = s["x"][a:a + 131_072].to(f64)
            mu = torch.einsum("ij->i", x) / d
            second = torch.einsum("ij,ij->i", x - mu[:, None], x - mu[:, None]) / d
            r = 1 / torch.sqrt(second + s["eps"])
            out.append(torch.einsum("ij,i,j->ij", x - mu[:, None], r, s["gain"].to(f64)) + s["offset"].to(f64))
            means.append(mu)
            scales.append(r)
        return torch.cat(out), torch.cat(means), torch.cat(scales)
    if kind == "norm_backward":
        # y = gain * xhat + offset with xhat = (x - mean) * rstd; the Jacobian of xhat is rstd (I - 1 1^T / d - xhat xhat^T / d).
        gain, g_gain, g_offset, out = s["gain"].to(f64), torch.zeros(d, dtype=f64, device="cuda"), torch.zeros(d, dtype=f64, device="cuda"), []
        for a in range(0, n, 131_072):
            xhat = torch.einsum("ij,i->ij", s["x"][a:a + 131_072].to(f64) - s["mean"][a:a + 131_072, None].to(f64), s["rstd"][a:a + 131_072].to(f64))
            g = s["g_y"][a:a + 131_072].to(f64)
            g_gain += torch.einsum("ij,ij->j", g, xhat)
            g_offset += torch.einsum("ij->j", g)
            along = torch.einsum("ij,ij,j->i", g, xhat, gain) / d
            level = torch.einsum("ij,j->i", g, gain) / d
            out.append((torch.einsum("ij,j->ij", g, gain) - level[:, None] - torch.einsum("ij,i->ij", xhat, along)) * s["rstd"][a:a + 131_072, None].to(f64))
        return torch.cat(out), g_gain, g_offset
    classes = case["classes"]
    step = max(1, min(n, 100_000_000 // max(classes, d)))
    if kind == "head":
        qw, sw = s["q_w"][:, :d].to(f64), s["s_w"].to(f64)
        if n * classes > 600_000_000:
            return None
        out = torch.empty((n, classes), dtype=f64, device="cuda")
        for a in range(0, n, step):
            x = s["x"][a:a + step].to(f64)
            top = x.abs().max(dim=1).values
            # 127 x lies between two integers k and k + 1 times the row's largest value; halfway goes to the even one.
            k = torch.floor(127 * x / top.clamp(min=1e-300)[:, None])
            beyond = 2 * 127 * x - (2 * k + 1) * top[:, None]
            q = torch.where((beyond > 0) | ((beyond == 0) & (k.remainder(2) == 1)), k + 1, k)
            out[a:a + step] = torch.einsum("ij,kj->ik", q, qw) * (top.float().to(f64) / 127)[:, None] * sw
        return out
    W = s["W"].to(f64)
    loss, lse = torch.zeros(n, dtype=f64, device="cuda"), torch.zeros(n, dtype=f64, device="cuda")
    g_x, g_w = (torch.zeros((n, d), dtype=f64, device="cuda"), torch.zeros((classes, d), dtype=f64, device="cuda")) if kind == "loss_step" else (None, None)
    rows = torch.nonzero(s["labels"] >= 0)[:, 0]
    for a in range(0, rows.numel(), step):
        r = rows[a:a + step]
        x, y = s["x"][r].to(f64), s["labels"][r]
        z = torch.einsum("ij,kj->ik", x, W)
        lse[r] = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[r][:, None])
        loss[r] = lse[r] - z[torch.arange(r.numel(), device="cuda"), y]
        if g_x is not None:
            weight = s["g_loss"][r].to(f64)
            g_x[r] = (torch.einsum("ik,kj->ij", p, W) - W[y]) * weight[:, None]
            g_w += torch.einsum("ik,ij->kj", p, x * weight[:, None])
            g_w.index_add_(0, y, -x * weight[:, None])
    return (loss, lse) if g_x is None else (loss, lse, g_x, g_w)

"""Which rows an 8-bit product takes for which class rows, on a context without a device: columns that quantize_rows() added are no columns of either."""
import pytest
import torch

from paper_2210_13149_b200 import binding as B


class Library:
    """Notes the length of the rows that a product is called with."""

    def __init__(self):
        self.d = None

    def bigcn_quantize_rows(self, h, x, x_type, n, d, *rest):
        return 0

    def bigcn_quantized_product(self, h, x, x_type, s_x, n, d, *rest):
        self.d = d
        return 0

    def bigcn_destroy(self, h):
        pass


@pytest.fixture
def ctx():
    c = object.__new__(B.BiGCN)
    c.lib, c.h, c.device, c.stream = Library(), 1, torch.device("cpu"), None
    c._outs = lambda *wanted, used=(): [torch.zeros(w[0], dtype=w[2]) for w in wanted]
    c._scratch = lambda nbytes: None
    return c


def rows(n, d):
    return torch.zeros((n, d))


def test_rows_of_another_length_are_refused_where_the_class_rows_say_theirs(ctx):
    q_w, s_w = ctx.quantize_rows(rows(5, 602))
    assert q_w.shape == (5, 608) and q_w.columns == 602
    ctx.quantized_product(rows(3, 602), q_w, s_w)
    assert ctx.lib.d == 602
    for d in (593, 600, 601, 603, 608, 609, 16):
        with pytest.raises(ValueError, match="rows of %d for class rows of 602" % d):
            ctx.quantized_product(rows(3, d), q_w, s_w)
        q_x, s_x = ctx.quantize_rows(rows(3, d))
        with pytest.raises(ValueError, match="class rows of 602|rows of %d for" % d):
            ctx.quantized_product(q_x, q_w, s_w, s_x=s_x)
    q_x, s_x = ctx.quantize_rows(rows(3, 602))
    ctx.quantized_product(q_x, q_w, s_w, s_x=s_x)
    assert ctx.lib.d == 602


def test_a_cut_between_multiples_of_16_says_it_too(ctx):
    q_w, s_w = ctx.quantize_rows(rows(5, 602))
    cut = q_w[:, :602]
    ctx.quantized_product(rows(3, 602), cut, s_w)
    assert ctx.lib.d == 602
    with pytest.raises(ValueError):
        ctx.quantized_product(rows(3, 600), cut, s_w)
    q_x, s_x = ctx.quantize_rows(rows(3, 601))
    with pytest.raises(ValueError):
        ctx.quantized_product(q_x, cut, s_w, s_x=s_x)
    with pytest.raises(ValueError):
        ctx.quantized_product(q_x[:, :601], q_w, s_w, s_x=s_x)
    q_x, s_x = ctx.quantize_rows(rows(3, 602))
    for x in (q_x, q_x[:, :602], q_x[:2], q_x.clone()):
        for w in (q_w, cut, q_w[:4], q_w.clone()):
            ctx.quantized_product(x, w, s_w[:w.shape[0]], s_x=s_x[:x.shape[0]])
            assert ctx.lib.d == 602 or (ctx.lib.d == 608 and x.shape[1] == w.shape[1] == 608 and not hasattr(x, "columns") and not hasattr(w, "columns"))


def test_class_rows_that_do_not_say_their_length(ctx):
    """A matrix made elsewhere, or a part of one: any length that quantize_rows() would lay out so."""
    q_w, s_w = torch.zeros((5, 608), dtype=torch.int8), torch.zeros(5)
    for d in (593, 600, 602, 608):
        ctx.quantized_product(rows(3, d), q_w, s_w)
        assert ctx.lib.d == d
    for d in (592, 609):
        with pytest.raises(ValueError):
            ctx.quantized_product(rows(3, d), q_w, s_w)
    for d in (1, 16):
        ctx.quantized_product(rows(3, d), torch.zeros((5, 16), dtype=torch.int8), s_w)
        assert ctx.lib.d == d

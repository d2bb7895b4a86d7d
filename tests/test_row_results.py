"""Row operators beside the library's others: what compile refuses because a kernel could not read it, and what is computed of what it takes."""
import numpy as np
import pytest

from paper_2302_00282_b200 import binding as xb

B, F = xb.DTYPE_BF16, xb.DTYPE_F32


def compiled(build, batch=3, link=False, precision=xb.PRECISION_BF16_TENSOR):
    """The graph of ``build(graph)``, which gives its results as [(tensor id, type)]."""
    g = xb.Graph()
    for t, dtype in build(g):
        g.mark_output(t, dtype, xb.LAYOUT_NHWC)
    if link:
        g.link()
    g.compile(batch, precision)
    return g


def refusal(build, **kw):
    with pytest.raises(xb.XenosError) as e:
        compiled(build, **kw)
    return e.value.code


def rows_in(g, dtype=B, c=64, h=2, w=2):
    return g.add_input(dtype, xb.LAYOUT_NHWC, c, h, w)


def norm(g, x, c=64):
    return g.add_op(xb.OP_LAYERNORM, [x], weight=np.ones(c))


def product(g, x, c=64, n=21):
    return g.add_qmatmul(x, np.ones((n, c), np.int8), np.ones(n))


# ---- widths ------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("link", [False, True])
def test_concat_refuses_widths_that_are_not_whole_chunks(link):
    """A part of 21 channels would be copied in pieces of 8 to rows of 85: every operand counts, not the first alone."""
    def concat(order, n):
        def build(g):
            x = rows_in(g)
            parts = [x, product(g, x, n=n), x]
            return [(g.add_op(xb.OP_CONCAT, [parts[i] for i in order]), B)]
        return build
    for order in ((0, 1), (1, 0), (0, 2, 1), (0, 1, 2)):
        assert refusal(concat(order, 21), link=link) == xb.E_UNSUPPORTED
        g = compiled(concat(order, 24), link=link)
        assert [l["kind"] for l in g.plan()["launches"]].count("concat_part") == len(order)

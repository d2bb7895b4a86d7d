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


# ---- types -------------------------------------------------------------------------------------------------------------------
def conv(g, x, n=64, c=64):
    return g.add_op(xb.OP_CONV, [x], cout=n, k=1, weight=np.ones((n, c, 1, 1)))


F32_READERS = {
    "add": lambda g, x: (g.add_op(xb.OP_ADD, [norm(g, x), x]), B),
    "add, other order": lambda g, x: (g.add_op(xb.OP_ADD, [x, norm(g, x)]), B),
    "mul": lambda g, x: (g.add_op(xb.OP_MUL, [norm(g, x), x]), B),
    "mac": lambda g, x: (g.add_op(xb.OP_MAC, [norm(g, x), norm(g, x), x]), B),
    "concat": lambda g, x: (g.add_op(xb.OP_CONCAT, [norm(g, x), x]), B),
    "split": lambda g, x: (g.add_op(xb.OP_SPLIT, [x], cout=8, pad=8), B),
    "max pool": lambda g, x: (g.add_op(xb.OP_POOL_MAX, [x], k=2, stride=2), B),
    "average pool": lambda g, x: (g.add_op(xb.OP_POOL_AVG, [x], k=2, stride=2), B),
    "global pool": lambda g, x: (g.add_op(xb.OP_POOL_GLOBAL_AVG, [x]), F),
    "convolution": lambda g, x: (conv(g, x), B),
    "depthwise": lambda g, x: (g.add_op(xb.OP_CONV, [x], cout=64, k=3, pad=1, groups=64, weight=np.ones((64, 1, 3, 3))), B),
    "shortcut": lambda g, x: (g.add_op(xb.OP_ADD, [conv(g, norm(g, x)), x]), B),
    "shortcut convolution": lambda g, x: (g.add_op(xb.OP_ADD, [conv(g, norm(g, x)), conv(g, x)]), B),
}


@pytest.mark.parametrize("link", [False, True])
@pytest.mark.parametrize("reader", F32_READERS)
def test_f32_inputs_are_for_row_operators_alone(reader, link):
    """A residual stream kept in 32 bits would be read as pairs of bf16 values."""
    def build(dtype):
        def f(g):
            x = rows_in(g, dtype)
            return [(norm(g, x), F), F32_READERS[reader](g, x)]
        return f
    assert refusal(build(F), link=link) == xb.E_UNSUPPORTED
    compiled(build(B), link=link)


def test_f32_inputs_of_row_operators_and_f32_images_stay():
    def rows(g):
        x = rows_in(g, F)
        y = norm(g, x)
        return [(product(g, x, n=24), F), (g.add_logprob(x)[1], F), (g.add_op(xb.OP_ADD, [y, norm(g, x)]), B)]
    assert len(compiled(rows, link=True).plan()["launches"]) >= 5

    def image(g):
        x = g.add_input(F, xb.LAYOUT_NCHW, 3, 8, 8)
        y = g.add_op(xb.OP_CONV, [x], cout=64, k=3, pad=1, weight=np.ones((64, 3, 3, 3)))
        return [(norm(g, y), B)]
    compiled(image, link=True)


@pytest.mark.parametrize("link", [False, True])
def test_f32_vector_outputs_are_read_by_row_operators_alone(link):
    """A global average that is an output of the graph lies in the caller's memory as fp32; a fully connected layer reads bf16."""
    def head(kind):
        def build(g):
            v = g.add_op(xb.OP_POOL_GLOBAL_AVG, [rows_in(g)])
            y = g.add_op(xb.OP_FC, [v], cout=8, k=1, weight=np.ones((8, 64))) if kind == "fc" else product(g, v) if kind == "product" else norm(g, v)
            return [(v, F), (y, F)]
        return build
    assert refusal(head("fc"), link=link) == xb.E_UNSUPPORTED
    compiled(head("product"), link=link)
    compiled(head("norm"), link=link)


# ---- vectors of any width ----------------------------------------------------------------------------------------------------
def picked(g, v, which, c=64):
    """An 8-bit product that picks channels.  (Rows of small whole numbers and one 127 keep their values: the rows' scale is 1.)"""
    w = np.zeros((len(which), c), np.int8)
    w[np.arange(len(which)), which] = 1
    return g.add_qmatmul(v, w, np.ones(len(which)))


def whole_rows(batch, key, c=64):
    rng = np.random.default_rng(key)
    x = rng.integers(-15, 16, (batch, c)).astype(np.float64)
    x[:, 0] = 127
    return x


def elementwise(kind, parts):
    """In fp32, rounded after the product."""
    a, b, *c = (p.astype(np.float32) for p in parts)
    return np.maximum(a + b, 0) if kind == "add, relu" else a + b if kind == "add" else a * b if kind == "mul" else a * b + c[0]


KINDS = {"add": (xb.OP_ADD, 2), "add, relu": (xb.OP_ADD, 2), "mul": (xb.OP_MUL, 2), "mac": (xb.OP_MAC, 3)}


def vector_case(kind, n, batch, finish):
    """finish(graph, element-wise result of vectors of n channels that products picked) -> results; the parts' values."""
    code, operands = KINDS[kind]
    which = [1 + (np.arange(n) * (3 + 2 * i) + i) % 63 for i in range(operands)]

    def build(g):
        v = g.add_op(xb.OP_POOL_GLOBAL_AVG, [g.add_input(B, xb.LAYOUT_NHWC, 64, 1, 1)])
        parts = [picked(g, v, w) for w in which]
        return finish(g, g.add_op(code, parts, act=xb.ACT_RELU if kind.endswith("relu") else xb.ACT_NONE))
    x = whole_rows(batch, n * 100 + batch)
    return build, x, elementwise(kind, [x[:, w] for w in which])


@pytest.mark.gpu
@pytest.mark.parametrize("n,batch", [(1, 1), (5, 1), (21, 1), (21, 3), (21, 8), (24, 3), (63, 7), (63, 33)])
@pytest.mark.parametrize("kind", KINDS)
def test_elementwise_vectors_of_any_width(kind, n, batch):
    """Batch x width need not be whole chunks of 8: the last elements are computed, too (a workspace starts as NaN)."""
    from row_util import Rows, rounded, to_device

    def finish(g, y):
        return [(g.add_qmatmul(y, np.eye(n, dtype=np.int8), np.ones(n)), n, "f32")]
    build, x, want = vector_case(kind, n, batch, finish)
    got, = Rows(build, batch).run([to_device(x, "bf16")], batch)
    want = rounded(want, "bf16")
    # the reader rounds each row to 127 steps of its largest magnitude: half a step, and the scale's rounding
    step = np.abs(want).max(axis=1, keepdims=True) / 127
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= step * (0.5 + 127 * 4 * 2.0 ** -24)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,batch", [(1, 1), (21, 3), (24, 5), (63, 33)])
@pytest.mark.parametrize("kind", KINDS)
def test_elementwise_vector_outputs_are_fp32(kind, n, batch):
    """A vector output is F32 whatever operator it comes from: the sum or product of bf16 operands, not rounded again."""
    from row_util import Rows, to_device
    build, x, want = vector_case(kind, n, batch, lambda g, y: [(y, n, "f32")])
    got, = Rows(build, batch).run([to_device(x, "bf16")], batch)
    assert np.array_equal(got, want)


@pytest.mark.gpu
def test_residual_sum_of_a_vector_leaves_as_fp32():
    """add(layernorm(v), v) is an output, and row operators read it as fp32."""
    from row_util import Rows, assert_within, rounded, to_device
    from oracle import rows as oracle
    rng = np.random.default_rng(5)
    x = rounded(rng.standard_normal((9, 64)) * 2, "bf16")

    def build(outputs):
        def f(g):
            v = g.add_op(xb.OP_POOL_GLOBAL_AVG, [g.add_input(B, xb.LAYOUT_NHWC, 64, 1, 1)])
            y = norm(g, v)
            if not outputs:
                return [(y, 64, "f32")]
            s = g.add_op(xb.OP_ADD, [y, v])
            return [(s, 64, "f32"), (norm(g, s), 64, "f32")]
        return f
    # (the layer norm's result as the add reads it: rounded to bf16, the same value as its fp32 output rounded here)
    y, = Rows(build(False), 9).run([to_device(x, "bf16")], 9)
    s, z = Rows(build(True), 9).run([to_device(x, "bf16")], 9)
    assert np.array_equal(s, (rounded(y, "bf16").astype(np.float32) + x.astype(np.float32)).astype(np.float64))
    want = oracle.layernorm(s, np.ones(64), np.zeros(64), 1e-5)
    rstd = 1 / np.sqrt(s.var(axis=1, keepdims=True) + 1e-5)
    assert_within(z, want, 2.0 ** -24 * np.abs(want) + 64 * 2.0 ** -24 * np.abs(s).max(axis=1, keepdims=True) * rstd)


# ---- numbers of rows ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("h,w,batch", [(65536, 65537, 1), (65536, 65536, 1), (46341, 46341, 3), (32769, 32768, 1), (32768, 16385, 2), (1 << 30, 3, 1)])
def test_more_than_2_to_30_rows_are_refused(h, w, batch):
    """Also where their number passes 32 bits: 65536 x 65537 rows are not 65536."""
    for build in (lambda g, x: norm(g, x, 1), lambda g, x: product(g, x, 1, 1), lambda g, x: g.add_logprob(x)[1]):
        assert refusal(lambda g: [(build(g, rows_in(g, F, 1, h, w)), F)], batch=batch) == xb.E_UNSUPPORTED
    compiled(lambda g: [(norm(g, rows_in(g, F, 1, 32768, 32768 // batch), 1), F)], batch=batch)


# ---- one order of a row's sums -----------------------------------------------------------------------------------------------
def normal_rows(rows, c, kind, key):
    from row_util import rounded
    rng = np.random.default_rng(key)
    return rounded(rng.standard_normal((rows, c)) * np.exp(0.5 * rng.standard_normal(c)) + 0.5, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c,kind", [
    (12000, 264, "bf16"), (9000, 512, "bf16"), (5003, 1032, "bf16"), (3700, 2048, "bf16"), (2400, 4096, "bf16"), (1300, 5000, "bf16"), (700, 12000, "bf16"), (300, 60, "bf16"),
    (300, 192, "bf16"), (3000, 333, "bf16"), (9600, 333, "bf16"), (3000, 1111, "bf16"), (5000, 1111, "bf16"), (2401, 4095, "bf16"), (900, 5001, "bf16"), (1250, 5001, "bf16"),
    (620, 9001, "bf16"), (300, 61, "bf16"), (40, 20001, "bf16"),
    (12000, 264, "f32"), (5003, 1032, "f32"), (2400, 2048, "f32"), (1300, 4096, "f32"), (700, 8000, "f32"), (100, 9000, "f32"), (3000, 333, "f32"), (777, 1111, "f32"), (300, 4095, "f32"),
    (300, 6001, "f32")])
def test_link_of_norm_and_product_changes_no_bit(rows, c, kind):
    """The sums of a row have one order, whichever kernel takes it: rows of the 8-bit values, scales and products are equal bit for bit."""
    from row_util import Rows, to_device
    rng = np.random.default_rng(c)
    gamma, beta = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32), (0.1 * rng.standard_normal(c)).astype(np.float32)
    w, s = rng.integers(-127, 128, (24, c)).astype(np.int8), (0.002 + 0.001 * rng.random(24)).astype(np.float32)
    x = to_device(normal_rows(rows, c, kind, rows), kind)

    def build(g):
        t = g.add_input(F if kind == "f32" else B, xb.LAYOUT_NHWC, c, 1, 1)
        return [(g.add_qmatmul(g.add_op(xb.OP_LAYERNORM, [t], weight=gamma, bias=beta), w, s), 24, "f32")]
    linked, plain = Rows(build, rows, link=True), Rows(build, rows)
    assert [ch["kind"] for ch in linked.g.plan()["chains"]] == ["norm_qmatmul"]
    assert [l["kind"] for l in plain.g.plan()["launches"]] == ["rows", "rows", "q8"]
    (a,), (b,) = linked.run([x], rows), plain.run([x], rows)
    assert np.array_equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c,kind", [
    (12000, 264, "bf16"), (9000, 512, "bf16"), (5003, 1032, "bf16"), (3700, 2048, "bf16"), (2400, 4096, "bf16"), (1300, 5000, "bf16"), (700, 12000, "bf16"), (9600, 333, "bf16"),
    (5000, 1111, "bf16"), (2401, 4095, "bf16"), (1250, 5001, "bf16"), (620, 9001, "bf16"), (12000, 264, "f32"), (9000, 1000, "f32"), (2400, 2048, "f32"), (1300, 4096, "f32"), (700, 8000, "f32")])
def test_norm_of_a_row_does_not_depend_on_the_number_of_rows(rows, c, kind):
    """Enough rows for the CTAs that stay, and the first and last of them alone."""
    from row_util import Rows, to_device
    rng = np.random.default_rng(c)
    gamma, beta = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32), (0.1 * rng.standard_normal(c)).astype(np.float32)
    x = normal_rows(rows, c, kind, rows)

    def build(g):
        t = g.add_input(F if kind == "f32" else B, xb.LAYOUT_NHWC, c, 1, 1)
        return [(g.add_op(xb.OP_LAYERNORM, [t], weight=gamma, bias=beta), c, "f32")]
    r = Rows(build, rows)
    many, = r.run([to_device(x, kind)], rows)
    for part in (slice(0, 100), slice(rows - 3, rows)):
        few, = r.run([to_device(x[part], kind)], len(x[part]))
        assert np.array_equal(few, many[part])


# ---- plans -------------------------------------------------------------------------------------------------------------------
def test_plan_names_the_kernels_of_rows():
    """By length, type, number of rows and how rows leave."""
    def names(rows, c, dtype=B, link=False, build=norm):
        def f(g):
            x = rows_in(g, dtype, c, 1, 1)
            return [(product(g, norm(g, x, c), c, 8) if link else build(g, x, c), F)]
        return [l["kernel"] for l in compiled(f, batch=rows, link=link).plan()["launches"]]
    assert names(1, 1024) == ["row_kernel"] and names(100, 4096) == ["row_kernel"]
    assert names(16384, 4096) == ["row_stream_kernel"] and names(16384, 1024, F) == ["row_stream_kernel"]
    assert names(16384, 256) == ["row_kernel"] and names(40000, 8200, F) == ["row_kernel"]
    assert names(50, 1111) == ["row_odd_kernel"] and names(16384, 1111, F) == ["row_odd_kernel"]
    assert names(16384, 4095) == ["row_stream_odd_kernel"]
    assert names(50, 16392) == ["row_long_kernel"] and names(50, 20001) == ["row_long_kernel"]
    assert names(16384, 4096, link=True) == ["row_kernel", "q8_tc_kernel"]
    assert names(16384, 4095, link=True) == ["row_odd_kernel", "q8_tc_kernel"]
    assert names(40, 16300, build=lambda g, x, c: product(g, x, c, 8)) == ["row_odd_kernel", "q8_tc_kernel"]
    assert names(40, 16385, build=lambda g, x, c: product(g, x, c, 8)) == ["row_long_kernel", "q8_tc_kernel"]
    assert names(4, 64, build=lambda g, x, c: product(g, x, c, 8)) == ["q8_small_kernel"]


# ---- stored graphs -----------------------------------------------------------------------------------------------------------
def test_images_with_empty_maps_are_refused():
    """An image with a right checksum whose input has no rows: the launch would divide by their number."""
    g = xb.Graph()
    x = g.add_input(F, xb.LAYOUT_NHWC, 9001, 77, 79)
    g.mark_output(g.add_logprob(x)[1], F, xb.LAYOUT_NHWC)
    img = bytearray(g.save()[:-8])
    extent = (77).to_bytes(4, "little") + (79).to_bytes(4, "little")
    places = [i for i in range(len(img) - 7) if img[i:i + 8] == extent]
    assert len(places) == 2                                     # the scores' and the entropy's

    def stored(h):
        for i in places:
            img[i:i + 4] = h.to_bytes(4, "little")
        v = 1469598103934665603
        for c in img:
            v = (v ^ c) * 1099511628211 % (1 << 64)
        return bytes(img) + v.to_bytes(8, "little")
    xb.Graph.load(stored(78))
    with pytest.raises(xb.XenosError) as e:
        xb.Graph.load(stored(0))
    assert e.value.code == xb.E_INVALID


# ---- scores from the library's other heads -----------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("head", ["convolution", "depthwise", "fc", "long fc"])
@pytest.mark.parametrize("batch", [1, 3, 40])
def test_answers_read_fp32_scores_of_every_head(head, batch):
    """Scores that leave the graph and scores that only LOGPROB reads are the same fp32 values: global averages behind a convolution or a depthwise chain, linked
    or not, and fully connected layers, one with a reduction that is cut."""
    from row_util import Rows, to_device
    rng = np.random.default_rng(len(head) * 100 + batch)
    w, wd = rng.standard_normal((104, 64, 1, 1)) * 0.2, rng.standard_normal((64, 1, 3, 3)) * 0.3
    wf = rng.standard_normal((104, 2048 if head == "long fc" else 64)) * 0.1
    wide = rng.standard_normal((2048, 64, 1, 1)) * 0.2

    def build(scores):
        def f(g):
            x = rows_in(g, B, 64, 7, 7)
            if head == "depthwise":
                x = g.add_op(xb.OP_CONV, [x], cout=64, k=3, pad=1, groups=64, weight=wd, act=xb.ACT_RELU)
            if head in ("convolution", "depthwise"):
                z = g.add_op(xb.OP_POOL_GLOBAL_AVG, [g.add_op(xb.OP_CONV, [x], cout=104, k=1, weight=w, act=xb.ACT_RELU)])
            else:
                if head == "long fc":
                    x = g.add_op(xb.OP_CONV, [x], cout=2048, k=1, weight=wide, act=xb.ACT_RELU)
                z = g.add_op(xb.OP_FC, [g.add_op(xb.OP_POOL_GLOBAL_AVG, [x])], cout=104, k=1, weight=wf)
            lp, ent, ids, tops = g.add_logprob(z, None, 4)
            return [(ids, 4, "i32"), (tops, 4, "f32"), (ent, 1, "f32")] + ([(z, 104, "f32")] if scores else [])
        return f
    x = to_device(rng.standard_normal((batch, 7, 7, 64)), "bf16")
    for link in (False, True):
        *want, z = Rows(build(True), batch, link=link).run([x], batch)
        assert np.isfinite(z).all() and z.std() > 0.01
        order = np.argsort(-z, axis=1, kind="stable")[:, :4]
        assert np.array_equal(want[0], order)
        for u, v in zip(Rows(build(False), batch, link=link).run([x], batch), want):
            assert np.array_equal(u, v)


# ---- the range of a layer norm -----------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("c", [64, 1111, 4096])
def test_norm_of_rows_beyond_the_range_of_squares(c):
    """Deviations whose squares are no fp32 numbers leave beta; rows whose sum is none leave NaN; the rows beside them are what they are alone."""
    from row_util import Rows, to_device
    rng = np.random.default_rng(c)
    beta = rng.standard_normal(c).astype(np.float32)
    x = rng.standard_normal((4, c))
    x[1] *= 1e25
    x[2] = 3e38

    def build(g):
        return [(g.add_op(xb.OP_LAYERNORM, [g.add_input(F, xb.LAYOUT_NHWC, c, 1, 1)], weight=np.ones(c), bias=beta), c, "f32")]
    r = Rows(build, 4)
    got, = r.run([to_device(x, "f32")], 4)
    assert np.array_equal(got[1], beta.astype(np.float64)) and np.isnan(got[2]).all()
    for i in (0, 3):
        alone, = r.run([to_device(x[i:i + 1], "f32")], 1)
        assert np.array_equal(alone[0], got[i]) and got[i].std() > 0.9


# ---- status ------------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_labels_outside_leave_the_arrival_counters_alone():
    """A label outside its row is an error of the caller's: the status is cleared, the counters that a pass behind it may be using are not.  A run that gave
    up clears both, and is reported before a label."""
    import torch
    from row_util import Rows, to_device
    c, rows = 20000, 3
    rng = np.random.default_rng(9)

    def build(g):
        t = g.add_input(F, xb.LAYOUT_NHWC, c, 1, 1)
        lp, ent, ids, tops = g.add_logprob(t, g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, 1, 1, 1), 4)
        return [(lp, 1, "f32"), (ids, 4, "i32"), (tops, 4, "f32")]
    r = Rows(build, rows)
    words = r.ws.view(torch.int32)              # no parameters: the status words come first, the counters behind 256 bytes
    assert not words[:64].any() and not words[64:64 + 2 * 148].any()
    x = to_device(rng.standard_normal((rows, c)), "f32")
    good, bad = (to_device(np.array(v, np.int32)[:, None], "i32") for v in ([5, -1, 19999], [5, 20000, -2]))
    want = r.run([x, good], rows)
    last = 64 + 2 * 148 - 1                     # the counter of a row that these runs do not have
    words[last] = 7

    def status():
        try:
            r.g.status(r.stream)
            return xb.XENOS_OK
        except xb.XenosError as e:
            return e.code
    got = r.run([x, bad], rows, status=False)
    assert status() == xb.E_BOUNDS and int(words[last]) == 7 and status() == xb.XENOS_OK
    assert got[0][0, 0] == want[0][0, 0] and np.isnan(got[0][1:]).all()
    for u, v in zip(r.run([x, good], rows), want):
        assert np.array_equal(u, v)
    r.run([x, bad], rows, status=False)
    r.g.selftest_wait_expiry(r.stream)
    assert status() == xb.E_TIMEOUT and int(words[last]) == 0 and status() == xb.XENOS_OK
    for u, v in zip(r.run([x, good], rows), want):
        assert np.array_equal(u, v)


# ---- host memory -------------------------------------------------------------------------------------------------------------
def test_compiled_8_bit_weights_are_held_twice():
    """What was given, for a stored graph, and what a binding uploads; no third time."""
    import os
    import subprocess
    import sys
    program = """
import numpy as np, resource
from paper_2302_00282_b200 import binding as xb
def graph(n, c):
    g = xb.Graph()
    x = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, 1, 1)
    g.mark_output(g.add_qmatmul(x, w[:n, :c], np.ones(n)), xb.DTYPE_F32, xb.LAYOUT_NHWC)
    g.compile(4, xb.PRECISION_BF16_TENSOR)
    return g
def now():
    return int(open('/proc/self/statm').read().split()[1]) * resource.getpagesize()
w = np.ones((16384, 8192), np.int8)
graph(8, 64)
before = now()
g = graph(16384, 8192)
print((now() - before) / w.nbytes)
"""
    out = subprocess.run([sys.executable, "-c", program], check=True, capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert 1.5 < float(out.stdout) < 2.5


# ---- images beside other inputs ----------------------------------------------------------------------------------------------
def conv_of(g, x, c, n=64, k=1):
    return g.add_op(xb.OP_CONV, [x], cout=n, k=k, pad=k // 2, weight=np.random.default_rng(c * 10 + k).standard_normal((n, c, k, k)) * 0.2)


def shortcut_of_image(dtype, c):
    def f(g):
        x, image = rows_in(g, B, 64, 4, 4), g.add_input(dtype, xb.LAYOUT_NCHW, c, 4, 4)
        return [(g.add_op(xb.OP_ADD, [conv_of(g, x, 64), conv_of(g, image, c)]), B)]
    return f


def expand_of_image(dtype, c):
    def f(g):
        image = g.add_input(dtype, xb.LAYOUT_NCHW, c, 4, 4)
        return [(g.add_op(xb.OP_CONCAT, [conv_of(g, image, c), conv_of(g, image, c, k=3)]), B)]
    return f


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("c", [3, 8, 64])
def test_links_leave_convolutions_of_images_alone(dtype, c):
    """A convolution that reads an NCHW image joins no chain as its shortcut or as one of two expansions: those kernels read NHWC."""
    for build in (shortcut_of_image, expand_of_image):
        linked, plain = compiled(build(dtype, c), link=True).plan(), compiled(build(dtype, c)).plan()

        def starts(p):
            return sorted(l["kernel"] for l in p["launches"] if l["kernel"] in ("gemm_chain_kernel", "stem3x3_kernel", "stem_tc_kernel"))
        assert starts(linked) == starts(plain) and starts(plain)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("c", [3, 8, 64])
def test_linked_shortcut_of_an_image(dtype, c):
    import torch
    from row_util import Rows, rounded, to_device
    rng = np.random.default_rng(c)
    kind = "f32" if dtype == F else "bf16"
    x, image = rounded(rng.standard_normal((3, 4, 4, 64)), "bf16"), rounded(rng.standard_normal((3, c, 4, 4)), kind)
    w = [rounded(np.random.default_rng(n * 10 + 1).standard_normal((64, n, 1, 1)) * 0.2, "bf16").reshape(64, n) for n in (64, c)]
    # (an fp32 image is rounded to bf16 in front of the product; half a step each, and one of the stored shortcut, of the result)
    a, b = x @ w[0].T, rounded(image, "bf16").transpose(0, 2, 3, 1) @ w[1].T
    tol = 2.0 ** -8 * (np.abs(a + b) + np.abs(b)) + 1e-4 * (np.abs(x) @ np.abs(w[0]).T)
    for link in (False, True):
        def build(g):
            return [(shortcut_of_image(dtype, c)(g)[0][0], 64, "bf16")]
        got, = Rows(build, 3, pixels=(4, 4), link=link).run([to_device(x, "bf16"), to_device(image, kind)], 3)
        slack = 0 if link else 2.0 ** -8 * np.abs(a)            # (unlinked: the other operand is stored, too)
        assert (np.abs(got.reshape(3, 4, 4, 64) - (a + b)) <= tol + slack).all()
    torch.cuda.synchronize()


@pytest.mark.parametrize("link", [False, True])
@pytest.mark.parametrize("reader", [r for r in F32_READERS if r not in ("convolution", "shortcut convolution")])
def test_nchw_inputs_are_for_dense_convolutions_alone(reader, link):
    """Their kernels would take the planes of an image for pixels; one pixel is the same memory either way."""
    def build(layout, side):
        def f(g):
            x = g.add_input(B, layout, 64, side, side)
            y = rows_in(g, B, 64, side, side)
            code = {"add": xb.OP_ADD, "add, other order": xb.OP_ADD, "mul": xb.OP_MUL, "concat": xb.OP_CONCAT}.get(reader)
            if code is not None:
                return [(g.add_op(code, [y, x] if reader != "add, other order" else [x, y]), B)]
            if reader == "mac":
                return [(g.add_op(xb.OP_MAC, [y, y, x]), B)]
            if reader == "shortcut":
                return [(g.add_op(xb.OP_ADD, [conv(g, y), x]), B)]
            return [F32_READERS[reader](g, x)]
        return f
    assert refusal(build(xb.LAYOUT_NCHW, 4), link=link) == xb.E_UNSUPPORTED
    compiled(build(xb.LAYOUT_NHWC, 4), link=link)
    if "pool" not in reader and reader != "depthwise":
        compiled(build(xb.LAYOUT_NCHW, 1), link=link)

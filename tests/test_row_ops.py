"""Layer normalisation, the product in 8-bit integers and log-probabilities: definitions, refusals, plans, and the kernels against
the definitions in 64 bits.

Tolerances.  A result is rounded to its type once: half_step |y|.  What is computed before that is fp32, u = 2^-24:
  norm     sums of n values by a tree (at most 32 + 5 + 4 roundings deep), quotient and square root: 64 u (|x|max rstd |gamma| + |beta|)
  product  the sum of products is exact (conversion u), two scales and a bias (3 u), each scale itself (u): 8 u (|sum sx sw| + |bias|)
  answers  a thread adds n / G terms, then a tree of 9 and up to 16 parts; a term e^d is off by 2^-22 (instruction) and by |d| 2^-23 (its
           argument), which e^d |d| < 1 makes 2^-23 of the sum per unit: (n / G + 64) u of the sum.  ln and the differences: u of their
           terms each."""
import numpy as np
import pytest

from oracle import rows as oracle
from paper_2302_00282_b200 import binding as xb
from row_util import Rows, assert_within, half_step, rounded, to_device

U = 2.0 ** -24
LOW = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38}


def rng_of(*key):
    """A generator of its own for every case, the same in every process."""
    return np.random.default_rng(sum((i + 1) * 7919 * ord(c) for i, c in enumerate(repr(key))) % (1 << 31))


def code(f):
    with pytest.raises(xb.XenosError) as e:
        f()
    return e.value.code


# ---- the definitions, pinned without themselves ------------------------------------------------------------------------------
def test_oracle_layernorm_closed_forms():
    x = np.array([[1.0, 3.0], [5.0, 5.0]])
    y = oracle.layernorm(x, [1, 1], [0, 0], 1e-12)
    assert np.allclose(y, [[-1, 1], [0, 0]])
    assert np.allclose(oracle.layernorm(x, [2, 3], [10, 20], 1e-12), [[8, 23], [10, 20]])


def test_oracle_quantise_ties_and_scales():
    # 127 x / a for a = 127 is x itself: halves go to the even neighbour
    q, s = oracle.quantise_rows(np.array([[127, 0.5, 1.5, -2.5, -127], [0, 0, 0, 0, 0]], float))
    assert q.tolist() == [[127, 0, 2, -2, -127], [0, 0, 0, 0, 0]] and s.tolist() == [1, 0]
    assert np.isnan(oracle.quantise_rows(np.array([[1, np.inf], [1, np.nan]]))[1]).all()


def test_oracle_qmatmul_by_hand():
    y = oracle.qmatmul(np.array([[127.0, -127.0]]), [[3, 1], [1, 3]], [0.5, 2.0], [1.0, 0.0], 0)
    assert np.allclose(y, [[0.5 * 127 * 2 + 1, -2.0 * 127 * 2]])
    assert np.allclose(oracle.qmatmul(np.array([[127.0, -127.0]]), [[3, 1], [1, 3]], [0.5, 2.0], None, 1), [[127.0, 0.0]])
    assert np.allclose(oracle.qmatmul(np.array([[127.0, -127.0]]), [[3, 1], [1, 3]], [0.5, 2.0], None, 2), [[6.0, 0.0]])


def test_oracle_logprob_closed_forms():
    x = np.array([[0, 0, 0, 0], [-np.inf, 2, -np.inf, 2], [-np.inf] * 4, [1, np.nan, 0, 0], [1, np.inf, 0, 0]])
    lp, ent, ids, tops = oracle.logprob(x, np.array([[1], [0], [0], [0], [-1]]), 3)
    assert np.allclose(lp[:2, 0], [-np.log(4), -np.inf]) and lp[2, 0] == -np.inf and np.isnan(lp[3, 0]) and lp[4, 0] == 0
    assert np.allclose(ent[:3, 0], [np.log(4), np.log(2), 0]) and np.isnan(ent[3:]).all()
    assert ids.tolist() == [[0, 1, 2], [1, 3, -1], [-1, -1, -1], [0, 2, 3], [1, 0, 2]]
    assert np.allclose(tops[1], [-np.log(2), -np.log(2), -np.inf]) and np.isneginf(tops[2]).all() and np.isnan(tops[3]).all()


# ---- refusals and plans, no GPU ----------------------------------------------------------------------------------------------
def test_refusals_at_the_call():
    g = xb.Graph()
    x = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, 16, 1, 1)
    labels = g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, 1, 1, 1)
    one = np.ones(16, np.float32)
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x])) == xb.E_INVALID                                  # no gamma
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x], weight=one, bn_eps=0.0)) == xb.E_INVALID
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x], weight=one, bn_eps=float("nan"))) == xb.E_INVALID
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x, x], weight=one)) == xb.E_INVALID
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x], weight=one * np.inf)) == xb.E_INVALID
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x], weight=one, act=xb.ACT_RELU)) == xb.E_INVALID
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x], weight=one, bn=(one, one, one, one))) == xb.E_INVALID
    assert code(lambda: g.add_op(xb.OP_QMATMUL, [x], weight=one)) == xb.E_UNSUPPORTED
    assert code(lambda: g.add_op(xb.OP_LOGPROB, [x])) == xb.E_UNSUPPORTED
    w8, w32, s = np.ones((4, 16), np.int8), np.ones((4, 16), np.float32), np.ones(4, np.float32)
    assert code(lambda: g.add_qmatmul(99, w8, s)) == xb.E_INVALID
    assert code(lambda: g.add_qmatmul(x, w8)) == xb.E_INVALID                                            # no scales
    assert code(lambda: g.add_qmatmul(x, w32, s)) == xb.E_INVALID                                        # scales beside floats
    assert code(lambda: g.add_qmatmul(x, w32 * np.nan)) == xb.E_INVALID
    assert code(lambda: g.add_qmatmul(x, w8, s * np.inf)) == xb.E_INVALID
    assert code(lambda: g.add_qmatmul(x, w8, s, bias=s * np.nan)) == xb.E_INVALID
    assert code(lambda: g.add_qmatmul(x, w8, s, act=7)) == xb.E_INVALID
    assert code(lambda: g.add_qmatmul(x, np.zeros((0, 16), np.int8), np.zeros(0))) == xb.E_SHAPE
    assert code(lambda: g.add_qmatmul(labels, np.ones((4, 1), np.int8), s)) == xb.E_UNSUPPORTED
    wide = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, 131073, 1, 1)
    assert code(lambda: g.add_qmatmul(wide, np.ones((1, 131073), np.int8), np.ones(1))) == xb.E_UNSUPPORTED
    with pytest.raises(ValueError):
        g.add_qmatmul(x, w8, np.ones(3))
    with pytest.raises(ValueError):
        g.add_op(xb.OP_LAYERNORM, [x], weight=one, bias=one[:15])
    assert code(lambda: g.add_op(xb.OP_LAYERNORM, [x], weight=one[:15])) == xb.E_SHAPE
    assert code(lambda: g.add_qmatmul(x, w8[:, :15], s)) == xb.E_SHAPE
    assert code(lambda: g.add_logprob(x, None, -1)) == xb.E_INVALID
    assert code(lambda: g.add_logprob(x, None, 33)) == xb.E_INVALID
    assert code(lambda: g.add_logprob(x, x, 1)) == xb.E_INVALID                                          # labels that are no labels
    assert code(lambda: g.add_logprob(x, 99, 1)) == xb.E_INVALID
    assert code(lambda: g.add_logprob(labels, None, 1)) == xb.E_UNSUPPORTED
    two = g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, 1, 2, 1)
    assert code(lambda: g.add_logprob(x, two, 1)) == xb.E_SHAPE
    lp, ent, ids, tops = g.add_logprob(x, labels, 2)
    assert g.add_logprob(x, None, 0)[0] is None
    assert code(lambda: g.add_op(xb.OP_RELU, [ent])) == xb.E_UNSUPPORTED                                 # results are results
    assert code(lambda: g.add_logprob(ent, None, 0)) == xb.E_UNSUPPORTED
    assert code(lambda: g.add_op(xb.OP_ADD, [labels, labels])) == xb.E_UNSUPPORTED
    assert code(lambda: g.mark_output(ids, xb.DTYPE_F32, xb.LAYOUT_NHWC)) == xb.E_INVALID
    assert code(lambda: g.mark_output(lp, xb.DTYPE_I32, xb.LAYOUT_NHWC)) == xb.E_INVALID
    g.mark_output(ids, xb.DTYPE_I32, xb.LAYOUT_NHWC)
    g.compile(4, xb.PRECISION_BF16_TENSOR)
    assert code(lambda: g.add_qmatmul(x, w8, s)) == xb.E_STATE
    assert code(lambda: g.add_logprob(x, labels, 2)) == xb.E_STATE


def _one(build, dtype=xb.DTYPE_BF16, layout=xb.LAYOUT_NHWC, c=64, h=1, w=1, precision=xb.PRECISION_BF16_TENSOR, out=xb.DTYPE_BF16, hw=None, batch=4,
         out_layout=None, link=False, split=False):
    g = xb.Graph(hw)
    x = g.add_input(dtype, layout, c, h, w)
    y = build(g, x)
    g.mark_output(y, out, (xb.LAYOUT_NHWC if precision == xb.PRECISION_BF16_TENSOR else xb.LAYOUT_NCHW) if out_layout is None else out_layout)
    if link:
        g.link()
    if split:
        g.split(y, parts_outc=2)
    g.compile(batch, precision)
    return g


def _norm(g, x, c=64):
    return g.add_op(xb.OP_LAYERNORM, [x], weight=np.ones(c), bias=np.zeros(c))


def _q8(g, x, c=64, n=24):
    return g.add_qmatmul(x, np.ones((n, c), np.int8), np.ones(n))


def test_refusals_at_compile():
    fp32 = dict(dtype=xb.DTYPE_F32, layout=xb.LAYOUT_NCHW, precision=xb.PRECISION_FP32_CUDA_CORE, out=xb.DTYPE_F32)
    _one(_norm, **fp32)
    assert code(lambda: _one(_norm, h=2, **fp32)) == xb.E_UNSUPPORTED                # channels are h * w apart
    assert code(lambda: _one(_q8, **fp32)) == xb.E_UNSUPPORTED
    assert code(lambda: _one(lambda g, x: g.add_logprob(x)[1], h=3, **fp32)) == xb.E_UNSUPPORTED
    _one(lambda g, x: g.add_logprob(x)[1], **fp32)
    assert code(lambda: _one(_norm, layout=xb.LAYOUT_NCHW, h=2, w=2)) == xb.E_UNSUPPORTED
    _one(_norm, layout=xb.LAYOUT_NCHW)
    assert code(lambda: _one(_norm, split=True)) == xb.E_BAD_SPLIT
    assert code(lambda: _one(_q8, split=True)) == xb.E_BAD_SPLIT
    assert code(lambda: _one(_norm, out=xb.DTYPE_F32, out_layout=xb.LAYOUT_NCHW)) == xb.E_UNSUPPORTED
    small = xb.HwInfo(4, 48 * 1024, 512, 1 << 20)
    assert code(lambda: _one(_q8, batch=64, hw=small)) == xb.E_UNSUPPORTED            # no room for two stages
    assert code(lambda: _one(lambda g, x: g.add_op(xb.OP_BATCHNORM, [_q8(g, x)], bn=(np.ones(24),) * 4))) == xb.E_UNSUPPORTED

    def f32_read_by_conv(g, x):
        y = _norm(g, x)
        g.mark_output(g.add_op(xb.OP_CONV, [y], cout=8, k=1, weight=np.ones((8, 64, 1, 1))), xb.DTYPE_BF16, xb.LAYOUT_NHWC)
        return y
    assert code(lambda: _one(f32_read_by_conv, out=xb.DTYPE_F32)) == xb.E_UNSUPPORTED

    def f32_vector_read_by_fc(g, x):
        y = _norm(g, g.add_op(xb.OP_POOL_GLOBAL_AVG, [x]))
        g.mark_output(g.add_op(xb.OP_FC, [y], cout=8, k=1, weight=np.ones((8, 64))), xb.DTYPE_F32, xb.LAYOUT_NHWC)
        return y
    assert code(lambda: _one(f32_vector_read_by_fc, out=xb.DTYPE_F32)) == xb.E_UNSUPPORTED
    # widths that the other bf16 operators do not take
    odd = lambda kind, **kw: code(lambda: _one(lambda g, x: g.add_op(kind, [_q8(g, x, n=21)], **kw), h=2))  # noqa: E731
    assert odd(xb.OP_CONV, cout=8, k=1, weight=np.ones((8, 21, 1, 1))) == xb.E_UNSUPPORTED
    assert odd(xb.OP_POOL_MAX, k=1) == xb.E_UNSUPPORTED
    _one(f32_read_by_conv, out=xb.DTYPE_BF16)


def test_plans_of_the_row_operators():
    def head(g, x):
        n = _norm(g, x)
        return _q8(g, n)
    kinds = lambda g: [(l["kind"]) for l in g.plan()["launches"]]  # noqa: E731
    assert kinds(_one(_q8, batch=16)) == ["q8_small"]
    assert kinds(_one(_q8, batch=17)) == ["rows", "q8"]
    assert kinds(_one(head, batch=17, link=True)) == ["rows", "q8"]
    assert kinds(_one(head, batch=16, link=True)) == ["rows", "q8_small"]
    g = _one(head, batch=17, link=True)
    assert [c["kind"] for c in g.plan()["chains"]] == ["norm_qmatmul"]
    g = _one(head, batch=17)
    assert [l["kind"] for l in g.plan()["launches"]] == ["rows", "rows", "q8"]
    # the link can be asked for where the rule would not make it
    def explicit(g, x):
        n = _norm(g, x)
        y = _q8(g, n)
        g.link([n, y])
        return y
    assert kinds(_one(explicit, batch=4)) == ["rows", "q8"]
    assert code(lambda: _one(lambda g, x: (lambda y: (g.link([y, g.add_op(xb.OP_RELU, [y])]), y)[1])(_norm(g, x)))) in (xb.E_UNSUPPORTED, xb.E_NOT_LINKABLE)
    # a large product is cut among pairs of CTAs, one of few tiles is not
    big = lambda batch: [l for l in _one(lambda g, x: _q8(g, x, 4096, 4096), c=4096, batch=batch).plan()["launches"] if l["kind"] == "q8"][0]  # noqa: E731
    assert big(8192)["pair"] == 1 and big(8192)["tile_n"] == 256
    assert big(100)["pair"] == 0
    # scores for LOGPROB alone stay fp32: twice the bytes of a bf16 tensor
    g = _one(lambda g, x: g.add_logprob(_q8(g, x), None, 2)[1], out=xb.DTYPE_F32, batch=256)
    p = g.plan()
    assert [t["bytes"] for t in p["tensors"] if t["c"] == 24 and not t["external"]] == [256 * 24 * 4]
    assert p == _one(lambda g, x: g.add_logprob(_q8(g, x), None, 2)[1], out=xb.DTYPE_F32, batch=256).plan()


def test_images_of_the_row_operators():
    def build(g, x):
        labels = g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, 2, 1, 1)
        rng = np.random.default_rng(1)
        y = g.add_qmatmul(_norm(g, x), rng.integers(-128, 128, (24, 64)).astype(np.int8), rng.random(24), bias=rng.random(24), act=xb.ACT_RELU6)
        lp, ent, ids, tops = g.add_logprob(y, labels, 3)
        g.mark_output(ids, xb.DTYPE_I32, xb.LAYOUT_NHWC)
        g.mark_output(lp, xb.DTYPE_F32, xb.LAYOUT_NHWC)
        return tops
    g = _one(build, out=xb.DTYPE_F32, batch=40, link=True)
    img = g.save()
    h, n = xb.Graph.load(img)
    assert h.plan_text() == g.plan_text() and n == g.plan()["workspace_bytes"] and h.save() == img
    # an image whose checksum is right but whose version does not go with its operators
    def fnv(b):
        v = 1469598103934665603
        for c in b:
            v = (v ^ c) * 1099511628211 % (1 << 64)
        return v.to_bytes(8, "little")
    old = bytearray(img[:-8]); old[8] = 1
    assert code(lambda: xb.Graph.load(bytes(old) + fnv(old))) == xb.E_INVALID
    assert img[8] == 2


def test_weights_in_floats_are_rounded_like_rows():
    rng = np.random.default_rng(3)
    w = rng.standard_normal((5, 37)).astype(np.float32)
    w[2] = 0
    q, s = oracle.quantise_rows(w)
    a, b = xb.Graph(), xb.Graph()
    for g, args in ((a, (w,)), (b, (q.astype(np.int8), s))):
        x = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, 37, 1, 1)
        g.mark_output(g.add_qmatmul(x, *args), xb.DTYPE_F32, xb.LAYOUT_NHWC)
    assert a.save() == b.save()


# ---- layer normalisation -----------------------------------------------------------------------------------------------------
def norm_case(rows, c, kind, out, seed, beta=True, mean=0.5, precision=xb.PRECISION_BF16_TENSOR, pixels=(1, 1)):
    rng = rng_of(rows, c, kind, out, seed)
    x = rng.standard_normal((rows, c)) * np.exp(0.5 * rng.standard_normal(c)) + mean * rng.standard_normal((rows, 1))
    gamma, bet = (1 + 0.3 * rng.standard_normal(c)).astype(np.float32), rng.standard_normal(c).astype(np.float32)
    batch = rows // (pixels[0] * pixels[1])

    def build(g):
        t = g.add_input(xb.DTYPE_F32 if kind == "f32" else xb.DTYPE_BF16, xb.LAYOUT_NHWC if precision else xb.LAYOUT_NCHW, c, *pixels)
        return [(g.add_op(xb.OP_LAYERNORM, [t], weight=gamma, bias=bet if beta else None, bn_eps=1e-5), c, out)]
    return build, batch, x, gamma, bet if beta else np.zeros(c)


def check_norm(got, x, gamma, beta, out):
    want = oracle.layernorm(x, gamma, beta, 1e-5)
    rstd = 1 / np.sqrt(x.var(axis=1, keepdims=True) + 1e-5)
    scale = np.abs(x).max(axis=1, keepdims=True) * rstd * np.abs(gamma) + np.abs(beta)
    assert_within(got, want, half_step(out) * np.abs(want) + 64 * U * scale)


@pytest.mark.gpu
@pytest.mark.parametrize("c", [1, 2, 7, 8, 56, 63, 64, 72, 128, 200, 256, 264, 512, 1000, 1024, 1111, 2048, 2056, 4096, 5000, 5001, 8192, 16384, 16392, 20001])
def test_norm_matches_the_definition(c):
    for rows, kind, out in ((37, "bf16", "bf16"), (1, "f32", "f32"), (5, "f32", "bf16"), (3, "bf16", "f32")):
        build, batch, x, gamma, beta = norm_case(rows, c, kind, out, 0)
        got, = Rows(build, batch).run([to_device(x, kind)], batch)
        check_norm(got, rounded(x, kind), gamma, beta, out)


@pytest.mark.gpu
@pytest.mark.parametrize("c,pixels", [(64, (7, 9)), (96, (5, 1)), (100, (3, 3))])
def test_norm_of_maps_without_beta(c, pixels):
    build, batch, x, gamma, beta = norm_case(pixels[0] * pixels[1] * 6, c, "bf16", "bf16", 1, beta=False, pixels=pixels)
    got, = Rows(build, batch, pixels).run([to_device(x, "bf16")], batch)
    check_norm(got, rounded(x, "bf16"), gamma, beta, "bf16")


@pytest.mark.gpu
def test_norm_of_rows_far_from_zero_and_of_constant_rows():
    build, batch, x, gamma, beta = norm_case(16, 777, "f32", "f32", 2, mean=0.0)
    x[:8] += 1000.0
    x[8] = 3.25
    x = rounded(x, "f32")
    got, = Rows(build, batch).run([to_device(x, "f32")], batch)
    check_norm(got, x, gamma, beta, "f32")
    assert np.array_equal(got[8], beta.astype(np.float64))


@pytest.mark.gpu
def test_norm_in_an_fp32_graph():
    build, batch, x, gamma, beta = norm_case(9, 333, "f32", "f32", 3, precision=xb.PRECISION_FP32_CUDA_CORE)
    got, = Rows(build, batch, precision=xb.PRECISION_FP32_CUDA_CORE).run([to_device(x, "f32")], batch)
    check_norm(got, rounded(x, "f32"), gamma, beta, "f32")


@pytest.mark.gpu
def test_norm_keeps_what_is_not_finite_in_its_row():
    build, batch, x, gamma, beta = norm_case(40, 72, "bf16", "bf16", 4)
    x = rounded(x, "bf16")
    clean, = Rows(build, batch).run([to_device(x, "bf16")], batch)
    bad = x.copy()
    bad[3, 5], bad[17, 0], bad[39, 71] = np.nan, np.inf, -np.inf
    got, = Rows(build, batch).run([to_device(bad, "bf16")], batch)
    hit = np.zeros(40, bool)
    hit[[3, 17, 39]] = True
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c", [(20001, 264), (9000, 512), (7500, 1000), (7301, 1024), (5003, 1032), (3700, 2048), (2500, 4000), (2400, 4096), (1300, 5000),
                                    (1200, 8192), (700, 16384), (601, 12000), (9500, 257), (9501, 1023), (4800, 2047), (2401, 4095), (1203, 8191), (602, 16383)])
def test_norm_of_many_rows(rows, c):
    """Enough rows for the CTAs that stay and walk over them; the last round of rows does not fill them."""
    for kind, out in (("bf16", "bf16"), ("f32", "f32")):
        build, batch, x, gamma, beta = norm_case(rows, c, kind, out, 5)
        got, = Rows(build, batch).run([to_device(x, kind)], batch)
        check_norm(got, rounded(x, kind), gamma, beta, out)


@pytest.mark.gpu
def test_rows_whose_offsets_pass_32_bits():
    """More than 2^31 elements: the last rows of a layer norm and of a row of scores."""
    import torch
    c, rows = 32768, 65535 + 4
    h = 3
    batch = -(-rows // h)
    rows = batch * h
    x = torch.empty((rows, c), dtype=torch.bfloat16, device="cuda")
    x[:-2] = 0
    tail = rng_of("far").standard_normal((2, c))
    x[-2:] = torch.from_numpy(tail).to(torch.bfloat16).cuda()
    gamma = np.ones(c, np.float32)

    def norm(g):
        t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, h, 1)
        return [(g.add_op(xb.OP_LAYERNORM, [t], weight=gamma), c, "bf16")]

    def answers(g):
        t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, h, 1)
        lp, ent, ids, tops = g.add_logprob(t, None, 3)
        return [(ent, 1, "f32"), (ids, 3, "i32"), (tops, 3, "f32")]
    xt = rounded(tail, "bf16")
    r = Rows(answers, batch, (h, 1))
    got = r.run([x], batch)
    check_lp([a[-2:] for a in got], xt, None, 3)
    r = Rows(norm, batch, (h, 1))
    y = torch.empty((rows + 1, c), dtype=torch.bfloat16, device="cuda")
    y[-1] = -77
    r.g.run(batch, [x.data_ptr()], [y.data_ptr()], r.stream)
    r.g.status(r.stream)
    check_norm(y[-3:-1].double().cpu().numpy(), xt, gamma, np.zeros(c), "bf16")
    assert bool((y[-1] == -77).all()) and not bool(y[0].any())


# ---- the product in 8-bit integers -------------------------------------------------------------------------------------------
def q8_case(rows, c, n, kind, out, act, bias, seed):
    rng = rng_of(rows, c, n, kind, out, act, seed)
    x = rng.standard_normal((rows, c)) * np.exp(0.5 * rng.standard_normal(c))
    w = rng.integers(-128, 128, (n, c)).astype(np.int8)
    s = (0.01 * (0.5 + rng.random(n))).astype(np.float32)
    b = rng.standard_normal(n).astype(np.float32) if bias else None

    def build(g):
        t = g.add_input(xb.DTYPE_F32 if kind == "f32" else xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, 1, 1)
        return [(g.add_qmatmul(t, w, s, bias=b, act=act), n, out)]
    return build, x, w, s, b


def check_q8(got, x, w, s, b, act, out):
    plain = oracle.qmatmul(x, w, s, None, 0)
    want = oracle.qmatmul(x, w, s, b, act)
    scale = np.abs(plain) + (0 if b is None else np.abs(b))
    assert_within(got, want, half_step(out) * np.abs(want) + 8 * U * np.where(np.isfinite(scale), scale, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c,n", [(1, 1, 1), (1, 16, 8), (1, 4096, 100), (2, 100, 33), (8, 128, 64), (8, 1111, 31), (9, 64, 17), (16, 1024, 1000),
                                      (16, 200, 1999), (17, 64, 32), (17, 1, 5), (100, 1000, 1000), (128, 128, 256), (129, 129, 257), (300, 1111, 1999),
                                      (513, 320, 96), (600, 300, 520), (2100, 520, 2056), (1500, 130, 3001), (40, 16500, 40), (5, 9000, 24), (3, 512, 6001), (1, 16384, 4800)])
def test_q8_matches_the_definition(rows, c, n):
    for kind, out, act, bias in (("bf16", "bf16", 0, True), ("f32", "f32", 1, False), ("bf16", "f32", 2, True), ("f32", "bf16", 0, False)):
        build, x, w, s, b = q8_case(rows, c, n, kind, out, act, bias, 0)
        got, = Rows(build, rows).run([to_device(x, kind)], rows)
        check_q8(got, rounded(x, kind), w, s, b, act, out)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c,n", [(2048, 4096, 4096), (3001, 2600, 2500), (2500, 4096, 2049)])
def test_q8_by_pairs_of_ctas(rows, c, n):
    for kind, out in (("bf16", "bf16"), ("f32", "f32")):
        build, x, w, s, b = q8_case(rows, c, n, kind, out, 0, True, 1)
        r = Rows(build, rows)
        assert [l["pair"] for l in r.g.plan()["launches"] if l["kind"] == "q8"] == [1]
        got, = r.run([to_device(x, kind)], rows)
        check_q8(got, rounded(x, kind), w, s, b, 0, out)
        # fewer rows than it was compiled for: another plan of tiles, the rows behind stay
        few = 1 + rows // 3
        got, = r.run([to_device(x[:few], kind)], few)
        check_q8(got, rounded(x[:few], kind), w, s, b, 0, out)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 40])
def test_q8_rounds_halves_to_even(rows):
    # 127 x / a with a = 127 2^e hits halves exactly; a = 254 / 2^k and 85 and 51 hit them through a quotient
    rng = rng_of("halves")
    x = np.zeros((rows, 256))
    for r in range(rows):
        a = [127.0, 254.0, 85.0, 51.0, 127 * 2.0 ** -130, 127 * 2.0 ** 100][r % 6]
        x[r] = rounded((rng.integers(-126, 126, 256) + 0.5) / 127 * a, "bf16")
        x[r, 0] = a
    w, s = np.eye(256, dtype=np.int8), np.ones(256, np.float32)

    for kind in ("bf16", "f32"):
        def build(g):
            t = g.add_input(xb.DTYPE_F32 if kind == "f32" else xb.DTYPE_BF16, xb.LAYOUT_NHWC, 256, 1, 1)
            return [(g.add_qmatmul(t, w, s), 256, "f32")]
        got, = Rows(build, rows).run([to_device(x, kind)], rows)
        q, sx = oracle.quantise_rows(rounded(x, kind))
        sx = sx.astype(np.float32).astype(np.float64)          # (the scale of a row near the smallest numbers has few digits)
        with np.errstate(divide="ignore", invalid="ignore"):
            assert np.array_equal(np.rint(got / sx[:, None]), q)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [7, 50])
def test_q8_rows_of_zeros_and_rows_that_are_not_finite(rows):
    build, x, w, s, b = q8_case(rows, 200, 40, "bf16", "bf16", 1, True, 2)
    x = rounded(x, "bf16")
    x[0] = 0
    x[2, 7], x[4, 199], x[5, 0] = np.nan, np.inf, -np.inf
    x[6] = LOW["bf16"]
    got, = Rows(build, rows).run([to_device(x, "bf16")], rows)
    with np.errstate(over="ignore", invalid="ignore"):
        want = oracle.qmatmul(x, w, s, b, 1)
    assert np.isnan(got[[2, 4, 5]]).all()
    assert np.array_equal(got[0], rounded(np.maximum(b, 0)[None].astype(np.float64), "bf16")[0])
    keep = [r for r in range(rows) if r not in (2, 4, 5, 6)]
    check_q8(got[keep], x[keep], w, s, b, 1, "bf16")
    big = np.abs(want[6]) < 3e38                                # (the others leave the range of bf16)
    assert np.allclose(got[6][big], want[6][big], rtol=2.0 ** -7)


@pytest.mark.gpu
def test_q8_largest_sums_do_not_overflow():
    # 131072 products of 127 * 128 with one sign
    w, s = np.full((8, 131072), -128, np.int8), np.ones(8, np.float32)

    def build(g):
        t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, 131072, 1, 1)
        return [(g.add_qmatmul(t, w, s), 8, "f32")]
    for rows in (1, 20):
        x = np.full((rows, 131072), 127.0)
        got, = Rows(build, rows).run([to_device(x, "bf16")], rows)
        assert (got == -127.0 * 128 * 131072).all()


# ---- log-probabilities -------------------------------------------------------------------------------------------------------
def lp_build(c, kind, n_labels, top, pixels=(1, 1), precision=xb.PRECISION_BF16_TENSOR):
    def build(g):
        t = g.add_input(xb.DTYPE_F32 if kind == "f32" else xb.DTYPE_BF16, xb.LAYOUT_NHWC if precision else xb.LAYOUT_NCHW, c, *pixels)
        labels = g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, n_labels, *pixels) if n_labels else None
        lp, ent, ids, tops = g.add_logprob(t, labels, top)
        return ([(lp, n_labels, "f32")] if n_labels else []) + [(ent, 1, "f32")] + ([(ids, top, "i32"), (tops, top, "f32")] if top else [])
    return build


def check_lp(got, x, labels, top):
    n = x.shape[1]
    group = 32 if n <= 2048 else 128 if n <= 8192 else 512
    lp, ent, ids, tops = oracle.logprob(x, labels, top)
    finite = np.where(np.isfinite(x), np.abs(x), 0)
    # |x - m| of what carries weight is below 100, and so are m and ln S in these inputs unless x itself is larger
    tol = (n / group + 64) * U + 4 * U * (finite.max(axis=1, keepdims=True) + 20)
    got = list(got)
    if labels is not None:
        g = got.pop(0)
        far = np.where(np.isfinite(lp), np.abs(lp), 0)
        assert_within(g, lp, tol + 2 * U * far)
    assert_within(got.pop(0), ent, tol * (1 + np.log(n)))
    if top:
        assert np.array_equal(got[0], ids)
        assert_within(got[1], tops, tol + 2 * U * np.where(np.isfinite(tops), np.abs(tops), 0))


def lp_input(rows, c, n_labels, seed, masked=0.0):
    rng = rng_of(rows, c, n_labels, seed)
    x = 3 * rng.standard_normal((rows, c))
    if masked:
        x[rng.random((rows, c)) < masked] = -np.inf
    labels = rng.integers(0, c, (rows, n_labels)).astype(np.int32) if n_labels else None
    if n_labels:
        labels[rng.random(labels.shape) < 0.2] = -1
    return x, labels


@pytest.mark.gpu
@pytest.mark.parametrize("c", [1, 2, 3, 7, 8, 9, 31, 100, 255, 1000, 1001, 2048, 2049, 5000, 8191, 8192, 8193, 20000, 50001, 131072, 200003])
def test_logprob_matches_the_definition(c):
    for rows, kind, n_labels, top, masked in ((1, "bf16", 1, 8, 0.0), (5, "f32", 3, 32, 0.3), (13, "bf16", 0, 5, 0.97), (29, "f32", 2, 0, 0.0), (1, "f32", 1, 1, 0.0)):
        if rows * c > 1 << 21:
            rows = max(2, (1 << 21) // c)
        x, labels = lp_input(rows, c, n_labels, 0, masked)
        ins = [to_device(x, kind)] + ([to_device(labels, "i32")] if n_labels else [])
        got = Rows(lp_build(c, kind, n_labels, top), rows).run(ins, rows)
        check_lp(got, rounded(x, kind), labels, top)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c", [(400, 1000), (600, 9000), (2, 40000), (148, 33000)])
def test_logprob_of_many_rows_twice(rows, c):
    x, labels = lp_input(rows, c, 1, 1)
    r = Rows(lp_build(c, "bf16", 1, 4), rows)
    ins = [to_device(x, "bf16"), to_device(labels, "i32")]
    first = r.run(ins, rows)
    check_lp(first, rounded(x, "bf16"), labels, 4)
    for _ in range(3):
        for a, b in zip(first, r.run(ins, rows)):
            assert np.array_equal(a, b)                        # no order of arrival in the results


@pytest.mark.gpu
@pytest.mark.parametrize("c", [40, 1500, 6000, 30000, 120000])
def test_logprob_ties_sorted_rows_and_plateaus(c):
    rng = rng_of("ties", c)
    x = np.zeros((10, c))
    x[1] = np.sort(rng.standard_normal(c))                      # every row's best are neighbours
    x[2] = x[1][::-1]
    x[3] = np.repeat(rng.standard_normal(c // 8 + 1), 8)[:c]
    x[4] = rng.integers(0, 3, c)
    x[5], x[6] = -0.0, np.where(np.arange(c) % 2, 0.0, -0.0)    # the two zeros are one value
    x[7] = -np.inf
    x[7, c // 2:] = 1.0
    x[8] = -20000.0
    x[9, : c // 3] = 5 + np.arange(c // 3) / c
    for kind in ("bf16", "f32"):
        got = Rows(lp_build(c, kind, 0, 32), 10).run([to_device(x, kind)], 10)
        check_lp(got, rounded(x, kind), None, 32)


@pytest.mark.gpu
@pytest.mark.parametrize("c", [17000, 24600, 65536, 131072])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_logprob_rows_of_several_parts(c, kind):
    """Two to sixteen CTAs share a row: as many answers as parts, fewer and more; parts without an entry, with all of the best, with equal ones."""
    x, _ = lp_input(8, c, 0, 7)
    sixteenth = c // 16
    x[1, -40:] += 50                                            # the best are all in the last part
    x[2] = -np.inf
    x[2, ::3 * sixteenth] = 1.0                                 # fewer entries than answers, far apart
    x[3] = 0.5
    x[4, ::sixteenth] = 90.0                                    # equal best entries in every part
    x[5] = np.linspace(4, -4, c)
    x[6, sixteenth:] = -np.inf                                  # entries in the first part only
    x[7, : c - 3] = -np.inf
    x = rounded(x, kind)
    dev = to_device(x, kind)
    for top in (1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 32):
        check_lp(Rows(lp_build(c, kind, 0, top), 8).run([dev], 8), x, None, top)


@pytest.mark.gpu
@pytest.mark.parametrize("c", [8, 1003, 4001, 60000])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_logprob_masks_and_values_that_are_not_finite(c, kind):
    x, labels = lp_input(12, c, 2, 2)
    x[0] = -np.inf                                              # nothing is left
    x[1] = -np.inf
    x[1, c - 1] = 2.0                                           # one entry is
    x[2, ::2] = LOW[kind]                                       # masks of the lowest value
    x[3] = LOW[kind]                                            # ... everywhere
    x[4, c // 2], x[5, 0], x[5, c - 1] = np.nan, np.inf, np.nan
    x[6] = np.nan
    x[7, 3] = np.inf
    x[8, 1:] = -np.inf
    x[8, 0] = LOW[kind]
    x[9] = 0
    x[9, 5] = 300.0
    labels[:, 0] = np.arange(12) % c
    labels[:, 1] = -1
    x = rounded(x, kind)
    got = Rows(lp_build(c, kind, 2, 6), 12).run([to_device(x, kind), to_device(labels, "i32")], 12)
    with np.errstate(over="ignore", invalid="ignore"):
        lp, ent, ids, tops = oracle.logprob(x, labels, 6)
    assert np.array_equal(got[2], ids)
    small = np.where(np.isfinite(x), np.where(np.abs(x) < 1e4, np.abs(x), 0), 0).max(axis=1, keepdims=True)
    tol = (c / 32 + 64) * U + 4 * U * (small + 20)
    for a, b in ((got[0], lp), (got[3], tops)):
        b = np.where(np.isfinite(b) & (b < -3.4e38), -np.inf, b)       # (below fp32)
        a = np.where(np.isfinite(a) & (a < -3.38e38) & np.isinf(b), -np.inf, a)
        assert_within(a, b, tol + 4 * U * np.where(np.isfinite(b), np.abs(b), 0))
    assert_within(got[1], ent, tol * (1 + np.log(c)))


@pytest.mark.gpu
def test_logprob_labels_outside_are_reported():
    x, labels = lp_input(6, 500, 3, 3)
    labels[2, 1], labels[4, 0], labels[5, 2] = 500, -2, 2 ** 31 - 1
    r = Rows(lp_build(500, "f32", 3, 2), 6)
    ins = [to_device(x, "f32"), to_device(labels, "i32")]
    bufs = r.buffers(6)
    got = r.run(ins, 6, bufs, status=False)
    assert code(lambda: r.g.status(r.stream)) == xb.E_BOUNDS
    r.g.status(r.stream)                                        # reported once
    check_lp(got, rounded(x, "f32"), labels, 2)
    good = np.clip(labels, -1, 499)
    check_lp(r.run([ins[0], to_device(good, "i32")], 6), rounded(x, "f32"), good, 2)


@pytest.mark.gpu
def test_logprob_in_an_fp32_graph_and_of_maps():
    x, labels = lp_input(7, 777, 1, 4)
    got = Rows(lp_build(777, "f32", 1, 3, precision=xb.PRECISION_FP32_CUDA_CORE), 7, precision=xb.PRECISION_FP32_CUDA_CORE).run(
        [to_device(x, "f32"), to_device(labels, "i32")], 7)
    check_lp(got, rounded(x, "f32"), labels, 3)
    x, labels = lp_input(4 * 15, 21, 1, 5)
    got = Rows(lp_build(21, "bf16", 1, 3, pixels=(5, 3)), 4, (5, 3)).run([to_device(x, "bf16"), to_device(labels, "i32")], 4)
    check_lp(got, rounded(x, "bf16"), labels, 3)


@pytest.mark.gpu
def test_logprob_computes_only_what_is_marked():
    x, labels = lp_input(9, 300, 2, 6)
    ref = Rows(lp_build(300, "f32", 2, 4), 9).run([to_device(x, "f32"), to_device(labels, "i32")], 9)
    for want in (0, 1, 2, 3):
        def build(g):
            t = g.add_input(xb.DTYPE_F32, xb.LAYOUT_NHWC, 300, 1, 1)
            o = g.add_logprob(t, g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, 2, 1, 1), 4)
            return [(o[want], (2, 1, 4, 4)[want], "i32" if want == 2 else "f32")]
        got, = Rows(build, 9).run([to_device(x, "f32"), to_device(labels, "i32")], 9)
        assert np.array_equal(got, ref[want])


# ---- together ----------------------------------------------------------------------------------------------------------------
def head_case(c, n, seed, act=0):
    rng = rng_of("head", c, n, seed)
    gamma, beta = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32), (0.1 * rng.standard_normal(c)).astype(np.float32)
    w, s = rng.integers(-127, 128, (n, c)).astype(np.int8), (0.002 + 0.001 * rng.random(n)).astype(np.float32)
    b = (0.1 * rng.standard_normal(n)).astype(np.float32)

    def build(marks=True):
        def f(g):
            t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, 1, 1)
            labels = g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, 1, 1, 1)
            y = g.add_qmatmul(g.add_op(xb.OP_LAYERNORM, [t], weight=gamma, bias=beta), w, s, bias=b)
            lp, ent, ids, tops = g.add_logprob(y, labels, 5)
            return [(lp, 1, "f32"), (ent, 1, "f32"), (ids, 5, "i32"), (tops, 5, "f32")] + ([(y, n, "f32")] if marks else [])
        return f
    return build, gamma, beta, w, s, b


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 16, 17, 300, 2100])
def test_head_linked_equals_unlinked_and_the_definition(rows):
    """A model's head: normalise, multiply in 8 bits, answer.  The link changes no bit; each stage equals the definition on what it reads."""
    c, n = 264, 2050
    build, gamma, beta, w, s, b = head_case(c, n, 0)
    rng = rng_of("head x", rows)
    x = rounded(2 * rng.standard_normal((rows, c)), "bf16")
    labels = rng.integers(0, n, (rows, 1)).astype(np.int32)
    ins = [to_device(x, "bf16"), to_device(labels, "i32")]
    linked, plain = Rows(build(), rows, link=True), Rows(build(), rows)
    a, p = linked.run(ins, rows), plain.run(ins, rows)
    for u, v in zip(a, p):
        assert np.array_equal(u, v)
    assert any(ch["kind"] == "norm_qmatmul" for ch in linked.g.plan()["chains"]) == (rows > 16)
    def norm(g):
        t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, 1, 1)
        return [(g.add_op(xb.OP_LAYERNORM, [t], weight=gamma, bias=beta), c, "bf16")]
    mid, = Rows(norm, rows).run(ins[:1], rows)
    check_norm(mid, x, gamma, beta, "bf16")
    check_q8(a[4], mid, w, s, b, 0, "f32")
    check_lp(a[:4], a[4], labels, 5)
    # scores that only LOGPROB reads: the same answers, from the workspace
    for u, v in zip(Rows(build(False), rows, link=True).run(ins, rows), a):
        assert np.array_equal(u, v)


@pytest.mark.gpu
def test_head_over_batches_streams_captures_images_and_the_built_in_scratch():
    import torch
    c, n, most = 128, 1000, 200
    build, gamma, beta, w, s, b = head_case(c, n, 1)
    r = Rows(build(), most, link=True)
    rng = rng_of("batches")

    def make(rows):
        return [to_device(2 * rng.standard_normal((rows, c)), "bf16"), to_device(rng.integers(0, n, (rows, 1)).astype(np.int32), "i32")]

    def alone(ins, rows):
        return Rows(build(), most, link=True).run(ins, rows)

    # other batches in turn, each twice (the second is recorded), with other buffers
    for rows in (200, 3, 3, 3, 129, 129, 1, 200):
        ins = make(rows)
        for u, v in zip(r.run(ins, rows), alone(ins, rows)):
            assert np.array_equal(u, v)
    # another stream than the one of the binding
    ins = make(77)
    want = alone(ins, 77)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    bufs = r.buffers(77)
    torch.cuda.synchronize()
    r.g.run(77, [t.data_ptr() for t in ins], [o.data_ptr() for o in bufs], side.cuda_stream)
    side.synchronize()
    for u, v in zip(r.read(bufs, 77), want):
        assert np.array_equal(u, v)
    # captured once, replayed on new values
    ins = make(50)
    bufs = r.buffers(50)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.g.run(50, [t.data_ptr() for t in ins], [o.data_ptr() for o in bufs], torch.cuda.current_stream().cuda_stream)
    for _ in range(2):
        new = make(50)
        for d, t in zip(ins, new):
            d.copy_(t)
        for o in bufs:
            o.fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(r.read(bufs, 50), alone(new, 50)):
            assert np.array_equal(u, v)
    # two bindings at work on two streams at once
    q = Rows(build(), most, link=True)
    ia, ib = make(200), make(150)
    wa, wb = alone(ia, 200), alone(ib, 150)
    ba, bb = r.buffers(200), q.buffers(150)
    torch.cuda.synchronize()
    for _ in range(20):
        r.g.run(200, [t.data_ptr() for t in ia], [o.data_ptr() for o in ba], r.stream)
        q.g.run(150, [t.data_ptr() for t in ib], [o.data_ptr() for o in bb], side.cuda_stream)
    torch.cuda.synchronize()
    for u, v in zip(r.read(ba, 200) + q.read(bb, 150), wa + wb):
        assert np.array_equal(u, v)
    # a stored graph, and the library's own workspace
    ins = make(200)
    want = r.run(ins, 200)
    loaded = Rows(r.outs, most, image=r.g.save())
    for u, v in zip(loaded.run(ins, 200), want):
        assert np.array_equal(u, v)
    bufs = r.buffers(200)
    for _ in range(2):
        r.g.run_builtin_scratch(200, [t.data_ptr() for t in ins], [o.data_ptr() for o in bufs], r.stream)
        for u, v in zip(r.read(bufs, 200), want):
            assert np.array_equal(u, v)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,c,mid", [(9, 264, 520), (40, 200, 333), (700, 512, 1000)])
def test_two_products_in_a_row(rows, c, mid):
    """norm -> product with ReLU -> norm -> product: both products' 8-bit rows lie in the same scratch."""
    rng = rng_of("two", rows)
    x = rounded(2 * rng.standard_normal((rows, c)), "bf16")
    g1, g2 = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32), (1 + 0.2 * rng.standard_normal(mid)).astype(np.float32)
    w1, w2 = rng.integers(-127, 128, (mid, c)).astype(np.int8), rng.integers(-127, 128, (c, mid)).astype(np.int8)
    s1, s2 = np.full(mid, 0.01, np.float32), np.full(c, 0.01, np.float32)

    def build(upto):
        def f(g):
            t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, 1, 1)
            a = g.add_op(xb.OP_LAYERNORM, [t], weight=g1)
            b = g.add_op(xb.OP_RELU, [g.add_qmatmul(a, w1, s1)])
            d = g.add_op(xb.OP_LAYERNORM, [b], weight=g2)
            y = g.add_qmatmul(d, w2, s2)
            return [((a, c), (b, mid), (d, mid), (y, c))[upto] + ("bf16",)]
        return f
    ins = [to_device(x, "bf16")]
    a, b, d, y = (Rows(build(i), rows).run(ins, rows)[0] for i in range(4))
    check_norm(a, x, g1, np.zeros(c), "bf16")
    check_q8(b, a, w1, s1, None, 1, "bf16")
    check_norm(d, b, g2, np.zeros(mid), "bf16")
    check_q8(y, d, w2, s2, None, 0, "bf16")
    r = Rows(build(3), rows, link=True)
    assert sum(ch["kind"] == "norm_qmatmul" for ch in r.g.plan()["chains"]) == (2 if rows > 16 else 0)
    for _ in range(3):
        assert np.array_equal(r.run(ins, rows)[0], y)


@pytest.mark.gpu
def test_batches_on_both_sides_of_the_kernels_rules():
    """A recorded pass whose kernels change with the batch: many rows, few rows, many again."""
    c, most = 4096, 2600
    rng = rng_of("rules")
    g1 = (1 + 0.2 * rng.standard_normal(c)).astype(np.float32)

    def build(g):
        t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, c, 1, 1)
        a = g.add_op(xb.OP_LAYERNORM, [t], weight=g1)
        lp, ent, ids, tops = g.add_logprob(g.add_op(xb.OP_LAYERNORM, [a], weight=g1), None, 3)
        return [(a, c, "f32"), (ent, 1, "f32"), (ids, 3, "i32"), (tops, 3, "f32")]
    r = Rows(build, most)
    for rows in (most, 30, 30, 30, most, most, 1, 1, 900, 900):
        x = rounded(2 * rng.standard_normal((rows, c)), "bf16")
        got = r.run([to_device(x, "bf16")], rows)
        check_norm(got[0], x, g1, np.zeros(c), "f32")
        z = oracle.layernorm(got[0], g1, np.zeros(c), 1e-5)
        lp, ent, ids, tops = oracle.logprob(z, None, 3)
        assert np.abs(got[1] - ent).max() < 1e-4 and np.abs(got[3] - tops).max() < 1e-4


@pytest.mark.gpu
def test_answers_of_an_image_classifier():
    """conv -> layer norm -> global average -> fc -> answers, and the same with an 8-bit head: the row operators beside the others."""
    import torch
    rng = rng_of("classifier")
    cw, fw, fb = rng.standard_normal((64, 16, 1, 1)) * 0.3, rng.standard_normal((100, 64)) * 0.2, rng.standard_normal(100) * 0.1

    def build(q8, scores):
        def f(g):
            t = g.add_input(xb.DTYPE_BF16, xb.LAYOUT_NHWC, 16, 6, 5)
            y = g.add_op(xb.OP_CONV, [t], cout=64, k=1, weight=cw)
            y = g.add_op(xb.OP_LAYERNORM, [y], weight=np.ones(64), bias=np.zeros(64))
            v = g.add_op(xb.OP_POOL_GLOBAL_AVG, [y])
            z = g.add_qmatmul(v, fw, bias=fb, act=xb.ACT_NONE) if q8 else g.add_op(xb.OP_FC, [v], cout=100, k=1, weight=fw, bias=fb)
            lp, ent, ids, tops = g.add_logprob(z, None, 5)
            return [(ids, 5, "i32"), (tops, 5, "f32"), (ent, 1, "f32")] + ([(z, 100, "f32")] if scores else [])
        return f
    for batch in (3, 40):
        x = to_device(rng.standard_normal((batch, 6, 5, 16)), "bf16")
        for q8 in (False, True):
            for link in (False, True):
                with_scores = Rows(build(q8, True), batch, link=link)
                ids, tops, ent, z = with_scores.run([x], batch)
                assert np.isfinite(z).all() and z.std() > 0.05
                check_lp([ent, ids, tops], z, None, 5)
                for u, v in zip(Rows(build(q8, False), batch, link=link).run([x], batch), (ids, tops, ent)):
                    assert np.array_equal(u, v)                 # the scores stay fp32 also inside
    torch.cuda.synchronize()

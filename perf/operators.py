"""What the row operators are measured on: layer normalisation, the product in 8-bit integers, and log-probabilities.

A program that uses one of them builds a graph with the operator once (its weights are packed then), compiles it for its
largest batch, binds a workspace and calls ``Graph.run`` with the rows and the results in device memory; that call is one
pass.  A row is the channels of one pixel of an NHWC map; a token is a row of a map of one pixel, and the batch counts tokens.
"""
import math

import torch

own = False


def listed():
    return [
        # One token's normalisation while a model answers: latency.
        dict(name="norm_token", op="norm", batch=1, h=1, w=1, c=1024, dtype="bf16"),
        # A feature map of the classifiers (56 x 56 x 64, batch 32), normalised over channels: very short rows.
        dict(name="norm_map_b32", op="norm", batch=32, h=56, w=56, c=64, dtype="bf16"),
        # A residual stream kept in 32 bits, of an odd length and an odd number of rows.
        dict(name="norm_ragged_f32", op="norm", batch=777, h=1, w=1, c=1111, dtype="f32"),
        # A long prompt's rows.
        dict(name="norm_prompt", op="norm", batch=16384, h=1, w=1, c=4096, dtype="bf16"),
        # One token against one layer's weights: the weights' bytes decide.
        dict(name="q8_token", op="q8", batch=1, h=1, w=1, c=4096, cout=4096, dtype="bf16", out="bf16", act=0, bias=False),
        # The classifier head (1024 features, 1000 classes) for 16 images, scores in 32 bits.
        dict(name="q8_classes_b16", op="q8", batch=16, h=1, w=1, c=1024, cout=1000, dtype="bf16", out="f32", act=0, bias=True),
        # A few hundred tokens, sizes that fill no tile, a 32-bit stream in, an activation.
        dict(name="q8_ragged", op="q8", batch=333, h=1, w=1, c=1111, cout=1999, dtype="f32", out="bf16", act=1, bias=True),
        # A long prompt against one wide layer: the tensor cores decide.
        dict(name="q8_prompt", op="q8", batch=8192, h=1, w=1, c=4096, cout=8192, dtype="bf16", out="bf16", act=0, bias=True),
        # The next token's distribution over a large vocabulary: one row.
        dict(name="answer_token", op="answer", batch=1, h=1, w=1, c=131072, labels=1, top=8, dtype="bf16", masked=0.0),
        # Scores of 1000 classes for a batch job of images: short rows in 32 bits.
        dict(name="answer_classes", op="answer", batch=4096, h=1, w=1, c=1000, labels=1, top=5, dtype="f32", masked=0.0),
        # A few candidates' scores under a mask (constrained answers), an odd vocabulary, several labels, one row with nothing left.
        dict(name="answer_masked", op="answer", batch=37, h=1, w=1, c=50001, labels=3, top=16, dtype="f32", masked=0.4),
        # Scoring a long text: every token's log-probability.
        dict(name="answer_text", op="answer", batch=4096, h=1, w=1, c=32768, labels=1, top=4, dtype="bf16", masked=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op, dtype = rng.choice(["norm", "q8", "q8", "answer", "answer"]), rng.choice(["bf16", "bf16", "f32"])
    # half of the lengths are multiples of 64, as they mostly are, the others any
    even = rng.random() < 0.5

    def length(lo, hi):
        n = _log_int(rng, lo, hi)
        return max(64, n // 64 * 64) if even else n

    if op == "norm":
        c = length(16, 16384)
        pixels = rng.choice([1, 1, 7, 14])
        return dict(op=op, batch=_log_int(rng, 1, max(1, min(32768, (1 << 26) // (c * pixels * pixels)))), h=pixels, w=pixels, c=c, dtype=dtype)
    if op == "q8":
        c, cout = length(32, 8192), length(8, 16384)
        batch = _log_int(rng, 1, min(8192, max(1, (1 << 38) // (c * cout))))
        return dict(op=op, batch=batch, h=1, w=1, c=c, cout=cout, dtype=dtype, out=rng.choice(["bf16", "bf16", "f32"]), act=rng.choice([0, 0, 1]),
                    bias=rng.random() < 0.5)
    c = length(10, 200000)
    return dict(op=op, batch=_log_int(rng, 1, min(8192, max(1, (1 << 26) // c))), h=1, w=1, c=c, labels=rng.choice([0, 1, 1, 2, 5]),
                top=rng.choice([0, 1, 4, 8, 20]) if c > 20 else 1, dtype=dtype, masked=rng.choice([0.0, 0.0, 0.3, 0.9]))


EPS = 1e-5


def _inputs(case, seed):
    rng = torch.Generator(device="cuda")
    rng.manual_seed(seed)
    b, h, w, c = case["batch"], case["h"], case["w"], case["c"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(shape, generator=rng, device="cuda")

    if case["op"] == "norm":
        # rows with a mean of their own and a few channels that are much larger than the others
        spread = torch.exp(0.7 * normal(c))
        x = normal(b, h, w, c) * spread + normal(b, h, w, 1)
        return dict(x=x.to(dtype), gamma=1 + 0.2 * normal(c), beta=0.1 * normal(c))
    if case["op"] == "q8":
        x = (normal(b, h, w, c) * torch.exp(0.5 * normal(c))).to(dtype)
        weight = normal(case["cout"], c) * math.sqrt(2.0 / c)
        scale = weight.abs().amax(dim=1) / 127
        return dict(x=x, weight=torch.round(weight / scale[:, None]).clamp(-127, 127).to(torch.int8), scale=scale,
                    bias=0.1 * normal(case["cout"]) if case["bias"] else None)
    x = 2.5 * normal(b, h, w, c)
    if case["masked"]:
        # entries that may not be chosen, and a last row with nothing left
        x[torch.rand(x.shape, generator=rng, device="cuda") < case["masked"]] = -math.inf
        if b > 4:
            x[-1] = -math.inf
    x = x.to(dtype)
    labels = None
    if case["labels"]:
        labels = torch.randint(0, c, (b, h, w, case["labels"]), generator=rng, device="cuda", dtype=torch.int32)
        # every eighth label is padding
        labels[torch.rand(labels.shape, generator=rng, device="cuda") < 0.125] = -1
    return dict(x=x, labels=labels)


def _graph(case, s):
    """The operator alone as a graph, with its result buffers."""
    from paper_2302_00282_b200 import binding as xb

    def buffer(n, dtype):
        return torch.empty((case["batch"], case["h"], case["w"], n), dtype=dtype, device="cuda")

    def host(t):
        return None if t is None else t.cpu().numpy()

    f32 = case["dtype"] == "f32"
    g = xb.Graph()
    x = g.add_input(xb.DTYPE_F32 if f32 else xb.DTYPE_BF16, xb.LAYOUT_NHWC, case["c"], case["h"], case["w"])
    ins, outs = [s["x"]], {}
    if case["op"] == "norm":
        y = g.add_op(xb.OP_LAYERNORM, [x], weight=host(s["gamma"]), bias=host(s["beta"]), bn_eps=EPS)
        outs["y"] = (y, buffer(case["c"], s["x"].dtype))
    elif case["op"] == "q8":
        y = g.add_qmatmul(x, host(s["weight"]), host(s["scale"]), bias=host(s["bias"]), act=case["act"])
        outs["y"] = (y, buffer(case["cout"], torch.float32 if case["out"] == "f32" else torch.bfloat16))
    else:
        labels = None
        if case["labels"]:
            labels = g.add_input(xb.DTYPE_I32, xb.LAYOUT_NHWC, case["labels"], case["h"], case["w"])
            ins.append(s["labels"])
        logprob, entropy, ids, tops = g.add_logprob(x, labels, top=case["top"])
        if case["labels"]:
            outs["logprob"] = (logprob, buffer(case["labels"], torch.float32))
        outs["entropy"] = (entropy, buffer(1, torch.float32))
        if case["top"]:
            outs["top_ids"] = (ids, buffer(case["top"], torch.int32))
            outs["top_logprobs"] = (tops, buffer(case["top"], torch.float32))
    kind = {torch.float32: xb.DTYPE_F32, torch.bfloat16: xb.DTYPE_BF16, torch.int32: xb.DTYPE_I32}
    for t, buf in outs.values():
        g.mark_output(t, kind[buf.dtype], xb.LAYOUT_NHWC)
    nbytes = g.compile(case["batch"], xb.PRECISION_BF16_TENSOR)
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    g.bind(ws.data_ptr(), ws.numel(), stream)
    return dict(graph=g, workspace=ws, stream=stream, ins=ins, outs={k: buf for k, (_, buf) in outs.items()})


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # the program's handle: the graph with its packed weights, bound to a workspace
        s["bound"] = _graph(case, s)
    s["case"] = case
    return s


def run(state):
    if own:
        b = state["bound"]
        b["graph"].run(state["case"]["batch"], [t.data_ptr() for t in b["ins"]], [t.data_ptr() for t in b["outs"].values()], b["stream"])
        return b["outs"]
    return {"norm": _norm, "q8": _q8, "answer": _answer}[state["case"]["op"]](state)


def _norm(s):
    x = s["x"].float()
    d = x - x.mean(dim=-1, keepdim=True)
    y = d * torch.rsqrt((d * d).mean(dim=-1, keepdim=True) + EPS) * s["gamma"] + s["beta"]
    return dict(y=y.to(s["x"].dtype))


def _q8(s):
    case = s["case"]
    x = s["x"].float()
    peak = x.abs().amax(dim=-1, keepdim=True)
    # (a quotient next to the middle of two whole numbers must round the right way: 64 bits)
    q = torch.round(127 * x.double() / torch.where(peak > 0, peak, 1).double()).float()
    y = (q @ s["weight"].float().T) * (peak / 127) * s["scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["act"]:
        y = torch.relu(y)
    return dict(y=y.to(torch.float32 if case["out"] == "f32" else torch.bfloat16))


def _answer(s):
    case, labels = s["case"], s["labels"]
    x = s["x"].float()
    peak = x.amax(dim=-1, keepdim=True)
    none = peak == -math.inf                      # nothing is left of the row
    d = x - torch.where(none, 0, peak)
    e = torch.exp(d)
    total = torch.where(none, 1, e.sum(dim=-1, keepdim=True))
    norm = torch.log(total)
    out = {}
    if labels is not None:
        lp = torch.gather(d, -1, labels.clamp(min=0).long()) - norm
        out["logprob"] = torch.where(labels < 0, 0, lp)
    out["entropy"] = norm - torch.where(e > 0, d * e, 0).sum(dim=-1, keepdim=True) / total
    if case["top"]:
        rest, ids = x.clone(), []
        for _ in range(case["top"]):
            i = rest.argmax(dim=-1, keepdim=True)     # (the first of equal values)
            ids.append(torch.where(torch.gather(rest, -1, i) == -math.inf, -1, i))
            rest.scatter_(-1, i, -math.inf)
        ids = torch.cat(ids, dim=-1)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprobs"] = torch.where(ids < 0, -math.inf, torch.gather(d, -1, ids.clamp(min=0)) - norm)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    x = s["x"].reshape(-1, case["c"]).to(torch.float64)
    rows = (case["batch"], case["h"], case["w"], -1)
    if case["op"] == "norm":
        var, mu = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        y = (x - mu) / torch.sqrt(var + EPS)
        return dict(y=torch.addcmul(s["beta"].double(), y, s["gamma"].double()).reshape(rows))
    if case["op"] == "q8":
        top = x.abs().max(dim=1, keepdim=True).values
        unit = top / 127.0
        whole = torch.where(top > 0, x * 127.0 / top, torch.zeros_like(x)).round()
        y = torch.matmul(whole, s["weight"].double().t()) * unit * s["scale"].double()[None, :]
        if s["bias"] is not None:
            y += s["bias"].double()
        return dict(y=(y.clamp(min=0.0) if case["act"] else y).reshape(rows))
    out = {}
    empty = torch.isneginf(x).all(dim=1, keepdim=True)
    lse = torch.logsumexp(x, dim=1, keepdim=True)
    if s["labels"] is not None:
        at = s["labels"].reshape(-1, case["labels"]).long()
        lp = x.gather(1, at.clamp(min=0)) - torch.where(empty, 0.0, lse)
        out["logprob"] = lp.masked_fill(at < 0, 0.0).reshape(rows)
    logp = (x - lse).masked_fill(torch.isneginf(x), -math.inf)
    out["entropy"] = -torch.special.xlogy(logp.exp(), logp.exp()).sum(dim=1, keepdim=True).reshape(rows) + 0.0
    if case["top"]:
        value, index = torch.sort(logp, dim=1, descending=True, stable=True)
        value, index = value[:, :case["top"]], index[:, :case["top"]]
        out["top_ids"] = index.masked_fill(torch.isneginf(value), -1).to(torch.int32).reshape(rows)
        out["top_logprobs"] = value.reshape(rows)
    return out


def work(case):
    """Every input read once, every output written once; two operations per multiply-accumulate."""
    rows, c = case["batch"] * case["h"] * case["w"], case["c"]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        return dict(bytes=2 * rows * c * es + 8 * c, flops=8.0 * rows * c)
    if case["op"] == "q8":
        n = case["cout"]
        return dict(bytes=rows * c * es + n * c + 4 * n * (2 if case["bias"] else 1) + rows * n * (4 if case["out"] == "f32" else 2), flops=2.0 * rows * c * n)
    return dict(bytes=rows * (c * es + 4 * (2 * case["labels"] + 1 + 2 * case["top"])), flops=5.0 * rows * c)

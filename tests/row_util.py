"""Helpers of the row operators' tests: one operator (or a head of several) as a graph on cuda:0, with sentinels behind its results."""
from __future__ import annotations

import numpy as np

from paper_2302_00282_b200 import binding as xb

KIND = {"f32": xb.DTYPE_F32, "bf16": xb.DTYPE_BF16, "i32": xb.DTYPE_I32}
GUARD = 3          # rows behind the last one, which no kernel may touch


def torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32}[name]


class Rows:
    """A compiled and bound graph; ``build(graph)`` gives its results as [(tensor id, channels, type)], in the order in which they are marked.
    With ``image``, a stored graph, ``build`` is that list itself."""

    def __init__(self, build, batch, pixels=(1, 1), precision=xb.PRECISION_BF16_TENSOR, link=False, image=None):
        import torch
        self.g = xb.Graph() if image is None else xb.Graph.load(image)[0]
        self.h, self.w = pixels
        self.outs = build(self.g) if image is None else build
        if image is None:
            for t, _, kind in self.outs:
                self.g.mark_output(t, KIND[kind], xb.LAYOUT_NHWC if precision == xb.PRECISION_BF16_TENSOR or kind == "i32" else xb.LAYOUT_NCHW)
            if link:
                self.g.link()
            n = self.g.compile(batch, precision)
        else:
            n = self.g.plan()["workspace_bytes"]
        self.ws = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        self.ws.fill_(0xFF)
        self.stream = torch.cuda.current_stream().cuda_stream
        self.g.bind(self.ws.data_ptr(), self.ws.numel(), self.stream)

    def buffers(self, batch):
        import torch
        rows = batch * self.h * self.w
        return [torch.full(((rows + GUARD) * c,), -77, dtype=torch_type(kind), device="cuda") for _, c, kind in self.outs]

    def run(self, ins, batch, bufs=None, status=True):
        bufs = self.buffers(batch) if bufs is None else bufs
        self.g.run(batch, [t.data_ptr() for t in ins], [b.data_ptr() for b in bufs], self.stream)
        if status:
            self.g.status(self.stream)
        return self.read(bufs, batch)

    def read(self, bufs, batch):
        rows = batch * self.h * self.w
        got = []
        for b, (_, c, kind) in zip(bufs, self.outs):
            a = (b.float() if kind != "i32" else b).cpu().numpy()
            assert (a[rows * c:] == -77).all(), "rows behind the last one were written"
            a = a[:rows * c].reshape(rows, c)
            got.append(a.astype(np.int64) if kind == "i32" else a.astype(np.float64))
        return got


def to_device(a, kind):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch_type(kind)).cuda()


def rounded(a, kind):
    """The values as the library sees them, in 64 bits."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch_type(kind)).double().numpy()


def half_step(kind):
    return 2.0 ** -8 if kind == "bf16" else 2.0 ** -24


def assert_within(got, want, tol):
    """NaN and infinities in the same places, the rest within tol element by element."""
    assert got.shape == want.shape
    assert (np.isnan(got) == np.isnan(want)).all()
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all() and not np.isinf(got[~inf]).any()
    ok = np.isfinite(want)
    over = np.abs(got - want)[ok] - np.broadcast_to(tol, want.shape)[ok]
    assert not ok.any() or over.max() <= 0, f"{over.max()} over the tolerance"

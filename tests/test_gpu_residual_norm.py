"""The norms on both sides of a residual against the formulas in 64 bits.

Tolerances.  One rounding of the result, u(T) of it, and `path(n)` (the roundings of the
longest fp32 path over n terms, see test_gpu_operators) times the sums of magnitudes
that a result is made of.  The second norm sees h as it is stored, so the reference
takes the kernel's own h there; h itself is checked on its own."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_operators import BF16, FP16, FP32, close, gap_untouched, gen, path, randn, same_bits, strided

pytestmark = pytest.mark.gpu
EPS = 1e-5
NAMES = ("dx", "dblock", "dgate", "dpost_weight", "dpost_bias", "dweight", "dbias")


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def statistics(x, layer):
    mean = x.mean(1) if layer else torch.zeros_like(x[:, 0])
    return mean, 1.0 / ((x - mean[:, None]).square().mean(1) + EPS).sqrt()


def wide(t, like, fill):
    return torch.full_like(like[:1], fill) if t is None else t.double()


def gates(gate, x):
    """A gate for every row."""
    if gate is None:
        return torch.ones_like(x)
    g = gate.double().reshape(-1, 1, x.shape[1])
    return g.expand(-1, x.shape[0] // g.shape[0], -1).reshape(x.shape)


class Case:
    def __init__(self, seed, rows, cols, dtype, param, kind="layer", post=True, groups=1, biases=True, scale=1.0, offset=0.0):
        g = self.g = gen(seed)
        self.kw = dict(kind=kind, post=post, scale=scale)
        self.layer, self.post, self.scale = kind == "layer", post, scale
        self.x, self.block = (randn(g, rows, cols) * 1.5 + offset).to(dtype), (randn(g, rows, cols) * 0.7 - 0.2 - offset).to(dtype)
        vector = lambda at, s: (at + s * randn(g, cols)).to(param)  # noqa: E731
        self.pw, self.pb = (vector(1, 0.2), vector(0, 0.3) if biases else None) if post else (None, None)
        self.w, self.b = vector(1, 0.2), vector(0, 0.3) if biases else None
        self.gate = None if not groups else (0.5 + 0.3 * randn(g, *((cols,) if groups == 1 else (groups, cols)))).to(param)
        self.dy, self.dh = (randn(g, rows, cols) * 0.3).to(dtype), (randn(g, rows, cols) * 0.2).to(dtype)

    def check_forward(self, **kw):
        h, y, stats = ops.residual_norm_forward(self.x, self.block, self.gate, self.pw, self.pb, self.w, self.b, **self.kw,
                                                eps=EPS, **kw)
        x, u, n = self.x.double(), self.block.double(), self.x.shape[1]
        e = path(n)
        pm, pr = statistics(u, self.layer) if self.post else (torch.zeros_like(x[:, 0]), torch.ones_like(x[:, 0]))
        spread = lambda t, r: (1.0 + t.abs().amax(1) * r * e)[:, None] if self.layer else torch.ones_like(t[:, :1])  # noqa: E731
        # a mean is a sum of terms whose magnitudes, not whose sum, its roundings are relative to:
        # |error| <= path(n) mean |x|, also where the mean itself is next to nothing
        hat, size = (u - pm[:, None]) * pr[:, None], (u.abs() + u.abs().mean(1, keepdim=True)) * pr[:, None] * spread(u, pr)
        pw, pb = wide(self.pw, x, 1.0), wide(self.pb, x, 0.0)
        v, size = hat * pw + pb, size * pw.abs() + pb.abs()
        g = gates(self.gate, x)
        want = self.scale * x + g * v
        close(h, want, e * (abs(self.scale) * x.abs() + g.abs() * size), "h")
        seen = h.double()
        m, r = statistics(seen, self.layer)
        w, b = wide(self.w, x, 1.0), wide(self.b, x, 0.0)
        size = (seen.abs() + seen.abs().mean(1, keepdim=True)) * r[:, None] * spread(seen, r)
        close(y, (seen - m[:, None]) * r[:, None] * w + b, e * (size * w.abs() + b.abs()), "y")
        for got, t, mean, rstd in ((stats[:2], u, pm, pr), (stats[2:], seen, m, r)):
            close(got[0], mean, e * t.abs().amax(1), "mean")
            close(got[1], rstd, e * rstd * (1.0 + (t.abs().amax(1) * rstd if self.layer else 0.0)), "rstd")
        return h, y, stats

    def check_backward(self, h, stats, dh=True, grads=None, **kw):
        dh = self.dh if dh else None
        args = dict(grads or {})
        before = {k: args[k].double().clone() for k in args} if kw.get("accumulate") else {}
        out = dict(zip(NAMES, ops.residual_norm_backward(self.dy, dh, h, self.block, stats, self.gate, self.pw, self.pb, self.w,
                                                         **self.kw, **args, **kw)))
        rows, n = h.shape
        e = path(n) + path(rows)
        pm, pr, m, r = (t.double()[:, None] for t in stats)
        dy, hd, block = self.dy.double(), h.double(), self.block.double()
        d = torch.zeros_like(dy) if dh is None else dh.double()
        w, pw, pb = wide(self.w, dy, 1.0), wide(self.pw, dy, 1.0), wide(self.pb, dy, 0.0)
        g = gates(self.gate, dy)
        mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
        inner = (lambda t: t - mean(t)) if self.layer else (lambda t: t)

        def through(q, q_size, hat, hat_size, rstd):
            """The norm's backward pass and the size of its terms."""
            value = rstd * (inner(q) - hat * mean(q * hat))
            return value, rstd * (q_size + mean(q_size) + hat_size * mean(q_size * hat_size))

        hat, hat_size = (hd - m) * r, (hd.abs() + m.abs()) * r
        t, size = through(dy * w, (dy * w).abs(), hat, hat_size, r)
        t, size = t + d, size + d.abs()
        bhat, bhat_size = (block - pm) * pr, (block.abs() + pm.abs()) * pr
        q, q_size = t * g * pw, size * (g * pw).abs()
        want = {"dx": (self.scale * t, abs(self.scale) * size)}
        want["dblock"] = through(q, q_size, bhat, bhat_size, pr) if self.post else (q, q_size)
        total = lambda value, size: (value.sum(0), size.sum(0))  # noqa: E731
        want["dweight"] = total(dy * hat, dy.abs() * hat_size)
        want["dbias"] = total(dy, dy.abs())
        want["dpost_weight"] = total(t * g * bhat, size * g.abs() * bhat_size)
        want["dpost_bias"] = total(t * g, size * g.abs())
        if self.gate is not None:
            u, u_size = (bhat * pw + pb, bhat_size * pw.abs() + pb.abs()) if self.post else (block, block.abs())
            by = lambda v: v.reshape(-1, rows // max(1, self.gate.numel() // n), n).sum(1).reshape(self.gate.shape)  # noqa: E731
            want["dgate"] = by(t * u), by(size * u_size)
        for name, got in out.items():
            if got is not None:
                value, size = want[name]
                if name in before:
                    value, size = value + before[name], size + before[name].abs()
                close(got, value, 4 * e * size, name)
        return out

    def check(self):
        h, y, stats = self.check_forward()
        out = self.check_backward(h, stats)
        assert (out["dgate"] is None) == (self.gate is None) and (out["dpost_weight"] is None) == (self.pw is None)
        assert (out["dpost_bias"] is None) == (self.pb is None) and out["dweight"] is not None
        assert (out["dbias"] is not None) == self.layer
        return h, y, stats, out


SHAPES = [(1, 1), (1, 4096), (3, 5), (5, 769), (64, 1024), (300, 768), (2047, 768), (33, 4096), (70, 4100), (9, 5120), (6, 8192), (3, 8200),
          (2, 20001), (1201, 96)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,param", [(BF16, BF16), (FP16, FP32), (FP32, FP32)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_forward_and_backward(rows, cols, dtype, param, kind):
    Case(rows + cols, rows, cols, dtype, param, kind, biases=kind == "layer", scale=0.75).check()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("groups", [0, 1, 4, 60])
@pytest.mark.parametrize("cols,dtype", [(512, BF16), (515, FP16), (1000, FP32), (4096, BF16)])
def test_gates_and_norms(kind, post, groups, cols, dtype):
    Case(groups + cols, 120, cols, dtype, FP32, kind, post, groups, biases=groups != 1).check()


@pytest.mark.parametrize("rows,groups", [(4096, 1), (4099, 1), (4096, 16), (6000, 3), (5000, 2500)])
def test_many_rows(rows, groups):
    Case(rows + groups, rows, 256, BF16, FP32, groups=groups).check()


@pytest.mark.parametrize("pad,offset", [(8, 0), (8, 8), (1, 0), (3, 5)])
@pytest.mark.parametrize("cols", [768, 767])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_strides_and_alignment(pad, offset, cols, dtype):
    c = Case(21, 19, cols, dtype, FP32)
    want = c.check()
    for name in ("x", "block", "dy", "dh"):
        setattr(c, name, strided(getattr(c, name), pad + len(name), offset))
    outs = [strided(torch.zeros(19, cols, dtype=dtype, device="cuda"), pad + i, offset) for i in range(4)]
    before = [t._base.clone() for t in outs]
    h, y, stats = c.check_forward(h=outs[0], y=outs[1])
    c.check_backward(h, stats, dx=outs[2], dblock=outs[3])
    assert all(gap_untouched(t, b) for t, b in zip(outs, before))
    w = torch.zeros(cols + 1, device="cuda")[1:].copy_(c.w)             # 4-byte aligned only
    c.w = w
    c.check()
    assert want[0].shape == h.shape


def test_in_place_broadcast_streams_and_stats():
    c = Case(22, 50, 1024, BF16, BF16, "rms")
    h, y, stats = c.check_forward()
    for name in ("x", "block"):
        t = getattr(c, name).clone()
        args = [t if name == k else getattr(c, k) for k in ("x", "block")]
        got = ops.residual_norm_forward(*args, c.gate, c.pw, c.pb, c.w, c.b, **c.kw, eps=EPS, h=t)
        assert got[0] is t and all(same_bits(a, b) for a, b in zip(got, (h, y, stats)))
    got = ops.residual_norm_forward(c.x, c.block, c.gate, c.pw, c.pb, c.w, c.b, **c.kw, eps=EPS, save_stats=False)
    assert got[2] is None and same_bits(got[1], y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.residual_norm_forward(c.x, c.block, c.gate, c.pw, c.pb, c.w, c.b, **c.kw, eps=EPS, stream=side)
    back = ops.residual_norm_backward(c.dy, c.dh, got[0], c.block, got[2], c.gate, c.pw, c.pb, c.w, **c.kw, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same_bits(a, b) for a, b in zip(got, (h, y, stats)))
    want = ops.residual_norm_backward(c.dy, c.dh, h, c.block, stats, c.gate, c.pw, c.pb, c.w, **c.kw)
    assert all((a is None and b is None) or same_bits(a, b) for a, b in zip(back, want))
    c.x, c.dy, c.dh = (t[:1].expand(50, 1024) for t in (c.x, c.dy, c.dh))          # row stride 0
    c.check()


def test_without_parameters_or_gradient_of_the_stream():
    c = Case(23, 37, 640, FP16, FP16, groups=0, biases=False)
    c.pw = c.w = None
    h, _, stats = c.check_forward()
    out = c.check_backward(h, stats, dh=False)
    assert out["dgate"] is None and out["dpost_weight"] is None and out["dweight"].dtype == FP16
    c = Case(24, 37, 640, BF16, BF16, "rms", post=False, groups=0, biases=False)
    h, _, stats = c.check_forward()
    none = {k: False for k in NAMES[2:]}
    out = c.check_backward(h, stats, grads=none)
    assert all(out[k] is None for k in none)


@pytest.mark.parametrize("rows,groups", [(120, 1), (3000, 4)])
@pytest.mark.parametrize("grad", [BF16, FP16, FP32])
def test_parameter_gradients_accumulate(rows, groups, grad):
    c = Case(25, rows, 768, BF16, FP32, groups=groups)
    h, _, stats = c.check_forward()
    shape = {"dgate": c.gate.shape}
    grads = {k: randn(c.g, *shape.get(k, (768,))).to(grad) for k in NAMES[2:]}
    c.check_backward(h, stats, grads=grads, accumulate=True)
    fresh = {k: torch.full_like(v, float("nan")) for k, v in grads.items()}
    c.check_backward(h, stats, grads=fresh)


def test_rows_far_from_zero():
    """The variance from centred values, however far the mean."""
    Case(26, 40, 2048, FP32, FP32, offset=300.0).check()


def test_rows_that_are_not_finite_stay_by_themselves():
    c = Case(27, 300, 768, BF16, FP32)
    h, y, stats = c.check_forward()
    c.block[7, 3], c.x[9, 5] = float("nan"), float("inf")
    h2, y2, _ = ops.residual_norm_forward(c.x, c.block, c.gate, c.pw, c.pb, c.w, c.b, **c.kw, eps=EPS)
    gone = torch.isnan(y2).all(1)
    assert gone.nonzero()[:, 0].tolist() == [7, 9] and same_bits(y2[~gone], y[~gone]) and same_bits(h2[~gone], h[~gone])


@pytest.mark.parametrize("rows", [0])
def test_no_rows(rows):
    c = Case(28, 4, 96, BF16, FP32)
    empty = c.x[:0]
    h, y, stats = ops.residual_norm_forward(empty, empty, c.gate, c.pw, c.pb, c.w, c.b, **c.kw)
    out = ops.residual_norm_backward(empty, empty, h, empty, stats, c.gate, c.pw, c.pb, c.w, **c.kw)
    assert h.shape == (0, 96) and all((g == 0).all() for g in out[2:])
    kept = torch.randn(96, device="cuda")
    dw = kept.clone()
    ops.residual_norm_backward(empty, None, h, empty, stats, c.gate, c.pw, c.pb, c.w, **c.kw, dweight=dw, dgate=False,
                               dpost_weight=False, dpost_bias=False, dbias=False, accumulate=True)
    assert torch.equal(dw, kept)


def test_gradients_against_differences():
    """fp32, steps of 2^-8 in one direction: the difference quotient is off by the third
    derivative's step^2 / 6 and by 2^-24 of sums of some thousand terms over the step."""
    c = Case(29, 12, 160, FP32, FP32, groups=3, scale=0.8)
    weights = [randn(c.g, 12, 160) for _ in range(2)]

    def value():
        x, u = c.x.double(), c.block.double()
        pm, pr = statistics(u, True)
        v = (u - pm[:, None]) * pr[:, None] * c.pw.double() + c.pb.double()
        h = c.scale * x + gates(c.gate, x) * v
        m, r = statistics(h, True)
        y = (h - m[:, None]) * r[:, None] * c.w.double() + c.b.double()
        return (h * weights[0]).sum() + (y * weights[1]).sum()

    h, y, stats = c.check_forward()
    c.dh, c.dy = weights[0], weights[1]
    out = c.check_backward(h, stats)
    for name, attribute in (("dx", "x"), ("dblock", "block"), ("dgate", "gate"), ("dpost_weight", "pw"), ("dpost_bias", "pb"),
                            ("dweight", "w"), ("dbias", "b")):
        at, way = getattr(c, attribute), randn(c.g, *getattr(c, attribute).shape)
        sides = []
        for sign in (1, -1):
            setattr(c, attribute, at.double() + sign * 2.0 ** -8 * way.double())
            sides.append(value())
        setattr(c, attribute, at)
        along = (out[name].double() * way.double()).sum()
        size = (out[name].double() * way.double()).norm() + 1
        assert ((sides[0] - sides[1]) / 2.0 ** -7 - along).abs() <= 2e-2 * size, name


def test_captured_and_replayed():
    c = Case(30, 500, 768, BF16, FP32, groups=5)
    h, y, stats = c.check_forward()
    grads = [torch.empty(5, 768, device="cuda")] + [torch.empty(768, device="cuda") for _ in range(4)]
    dx, dblock = torch.empty_like(h), torch.empty_like(h)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ops.residual_norm_forward(c.x, c.block, c.gate, c.pw, c.pb, c.w, c.b, **c.kw, eps=EPS, h=h, y=y, stats=stats)
            ops.residual_norm_backward(c.dy, c.dh, h, c.block, stats, c.gate, c.pw, c.pb, c.w, **c.kw, dx=dx, dblock=dblock,
                                       **dict(zip(NAMES[2:], grads)))
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        c.x.copy_(randn(c.g, 500, 768))
        c.dy.copy_(randn(c.g, 500, 768))
        graph.replay()
        got = [t.clone() for t in (h, y, stats, dx, dblock, *grads)]
        first = ops.residual_norm_forward(c.x, c.block, c.gate, c.pw, c.pb, c.w, c.b, **c.kw, eps=EPS)
        then = ops.residual_norm_backward(c.dy, c.dh, first[0], c.block, first[2], c.gate, c.pw, c.pb, c.w, **c.kw)
        assert all(same_bits(a, b) for a, b in zip(got, (*first, *then)))


@pytest.mark.parametrize("rows,cols,dtype,groups", [(3000, 256, BF16, 1), (2001, 768, FP16, 3), (900, 4096, BF16, 5), (700, 1024, FP32, 700), (500, 8192, BF16, 1)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_whose_copies_do_not_arrive(rows, cols, dtype, groups, kind):
    """NaN in the rows of the groups that gave up and in the gradients of parameters, all else as ever."""
    c = Case(31, rows, cols, dtype, FP32, kind, groups=groups)
    args = (c.x, c.block, c.gate, c.pw, c.pb, c.w, c.b)
    want = ops.residual_norm_forward(*args, **c.kw, eps=EPS)
    back = (c.dy, c.dh, want[0], c.block, want[2], c.gate, c.pw, c.pb, c.w)
    grads = ops.residual_norm_backward(*back, **c.kw)
    for unit in (-1, 0, 2):
        B.so_debug_set_operator_polls(0, unit)
        try:
            got = ops.residual_norm_forward(*args, **c.kw, eps=EPS)
            lost = ops.residual_norm_backward(*back, **c.kw)
        finally:
            B.so_debug_set_operator_polls(1 << 20)
        gone = torch.isnan(got[1]).all(1)
        assert gone.all() if unit < 0 else 0 < gone.sum() < rows
        for a, b in zip(got, want):
            a, b = (a, b) if a.shape[0] == rows else (a.t(), b.t())
            assert torch.isnan(a[gone]).all() and same_bits(a[~gone], b[~gone])
        gone = torch.isnan(lost[0]).all(1)
        assert gone.all() if unit < 0 else 0 < gone.sum() < rows
        for a, b in zip(lost[:2], grads[:2]):
            assert torch.isnan(a[gone]).all() and same_bits(a[~gone], b[~gone])
        assert torch.isnan(lost[2]).any()
        for name, a, b in zip(NAMES[3:], lost[3:], grads[3:]):
            # wide rows with biases have sums of their own, of which those of dy alone need nothing of what was lost
            if a is not None and cols == 8192 and name in ("dweight", "dbias"):
                assert same_bits(a, b)
            elif a is not None:
                assert torch.isnan(a).all()
    z = c.x.clone()
    B.so_debug_set_operator_polls(0, -1)
    try:
        ops.residual_norm_forward(z, *args[1:], **c.kw, eps=EPS, h=z)
    finally:
        B.so_debug_set_operator_polls(1 << 20)
    assert torch.isnan(z).all()

"""Layer norm, embedding and the losses on logits against plain implementations
in 64 bits, at the sizes, strides and masks where they can go wrong.

Tolerances.  u(T) is half an ulp of the output type (2^-8 bf16, 2^-11 fp16,
2^-24 fp32) and bounds the one rounding of the result; e = 2^-24 times the number
of roundings on the longest fp32 path bounds the rest, taken relative to the sum
of the absolute values of the terms (so cancellation is covered, not hidden).
Paths: a sum of n terms is split over at least 256 accumulators where n is large,
so n / 256 additions in a row, and at most 64 more for the trees, the partial sums
of blocks and the arithmetic of a term.  The hardware exponential is good to 2^-22
relative and gives 0 below 2^-126 (fp32 and bf16 results).  fp16 results below its
normal range are rounded to multiples of 2^-24."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, FP16: 2.0 ** -11, FP32: 2.0 ** -24}
FLOOR = {BF16: 2.0 ** -126, FP16: 2.0 ** -25, FP32: 2.0 ** -126}
E = 2.0 ** -24
EXP = 2.0 ** -22
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def path(n: int) -> float:
    return E * (n / 256 + 64)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def strided(t, pad, offset=0):
    """The same values in rows of `pad` more elements, `offset` elements into the buffer."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + offset,), 7.0, dtype=t.dtype, device="cuda")
    view = buf[offset:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


def gap_untouched(view, before):
    """The elements between the rows of a strided output are as they were."""
    base = view._base if view._base is not None else view
    flat, old = base.flatten(), before.flatten()
    hole = torch.ones_like(flat, dtype=torch.bool)
    hole.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return torch.equal(flat[hole], old[hole])


def close(got, want, slack, what):
    """|got - want| <= u |want| + floor + slack, NaN and infinities in the same places."""
    g = got.double()
    t = got.dtype
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(g), nan), f"{what}: NaN in other places"
    limit = torch.finfo(t).max * (1 + U[t])
    over = want.abs() > limit
    assert torch.equal(g[over], torch.sign(want[over]) * INF), f"{what}: infinities"
    ok = ~nan & ~over
    slack = slack.expand_as(want) if isinstance(slack, torch.Tensor) else torch.full_like(want, slack)
    err = (g - want).abs()[ok]
    tol = (U[t] * 1.0001 * want.abs() + FLOOR[t] * 1.0001 + slack)[ok]
    worst = (err / tol).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3f} of the tolerance"


def same_bits(a, b):
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


# --------------------------------------------------------------------------
# layer norm
# --------------------------------------------------------------------------

def norm_reference(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1.0 / ((c * c).mean(1, keepdim=True) + eps).sqrt()
    y = c * rstd
    if w is not None:
        y = y * w.double()
    if b is not None:
        y = y + b.double()
    return y, mean[:, 0], rstd[:, 0]


def check_norm_forward(x, w, b, eps=1e-5, **kw):
    y, mean, rstd = ops.layer_norm_forward(x, w, b, eps, **kw)
    want, m, r = norm_reference(x, w, b, eps)
    n = x.shape[1]
    top = x.double().abs().amax(1, keepdim=True)
    # the variance's relative error moves with the error of the mean against the spread
    spread = 1.0 + (top[:, 0] * r) * path(n)
    slack = path(n) * (1.0 if w is None else w.double().abs()) * (x.double().abs() + top) * r[:, None] * spread[:, None]
    slack = slack + path(n) * want.abs() + (0.0 if b is None else path(n) * b.double().abs())
    close(y, want, slack, "y")
    close(mean, m, path(n) * top[:, 0], "mean")
    close(rstd, r, path(n) * r * spread, "rstd")
    return y, mean, rstd


NORM_SHAPES = [(1, 1), (3, 2), (1, 768), (5, 769), (257, 768), (2047, 768), (7, 1000), (33, 1023), (64, 1024),
               (9, 1600), (600, 2048), (3, 4096), (301, 4096), (5, 4097), (4, 5120), (11, 8192), (2, 8193),
               (3, 16384), (2, 20001), (2, 65536)]


@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("dtype,param", [(BF16, BF16), (FP16, FP32), (FP32, FP32), (BF16, FP32), (FP16, FP16)])
def test_layer_norm_forward(rows, cols, dtype, param):
    g = gen(rows * 7 + cols)
    x = (randn(g, rows, cols) * 2 + 0.5).to(dtype)
    w, b = (1 + 0.2 * randn(g, cols)).to(param), (0.3 * randn(g, cols)).to(param)
    check_norm_forward(x, w, b)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("has_w,has_b", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("cols", [768, 515])
def test_layer_norm_without_weight_or_bias(dtype, has_w, has_b, cols):
    g = gen(5)
    x = randn(g, 37, cols).to(dtype)
    w = randn(g, cols) if has_w else None
    b = randn(g, cols).to(FP32) if has_b else None
    check_norm_forward(x, w, b)
    y, mean, rstd = ops.layer_norm_forward(x, w, b, save_stats=False)
    assert mean is None and rstd is None
    assert same_bits(y, ops.layer_norm_forward(x, w, b)[0])


@pytest.mark.parametrize("pad,offset", [(8, 0), (1, 0), (8, 8), (8, 1), (3, 5)])
@pytest.mark.parametrize("cols", [768, 767, 4096])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_layer_norm_strides_and_alignment(pad, offset, cols, dtype):
    g = gen(11)
    x = strided(randn(g, 19, cols).to(dtype), pad, offset)
    out = strided(torch.zeros(19, cols, dtype=dtype, device="cuda"), pad + 8, offset)
    w = torch.zeros(cols + 1, device="cuda")[1:].copy_(randn(g, cols))      # 4-byte aligned only
    before = out._base.clone()
    y, mean, rstd = check_norm_forward(x, w, None, out=out)
    assert gap_untouched(out, before)
    dy = strided(randn(g, 19, cols).to(dtype), pad + 2, offset)
    dx = strided(torch.zeros(19, cols, dtype=dtype, device="cuda"), pad + 1, offset)
    before = dx._base.clone()
    check_norm_backward(dy, x, mean, rstd, w, dx=dx)
    assert gap_untouched(dx, before)


def test_layer_norm_in_place_broadcast_rows_and_streams():
    g = gen(12)
    x = randn(g, 50, 1024).to(BF16)
    w = randn(g, 1024).to(BF16)
    y, mean, rstd = ops.layer_norm_forward(x, w, None)
    z = x.clone()
    ops.layer_norm_forward(z, w, None, out=z)
    assert same_bits(z, y)
    one = x[:1].expand(50, 1024)                     # row stride 0
    check_norm_forward(one, w, None)
    dy = randn(g, 1, 1024).to(BF16).expand(50, 1024)
    check_norm_backward(dy, x, mean, rstd, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2, _, _ = ops.layer_norm_forward(x, w, None, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert same_bits(y2, y)
    dy = dy.contiguous()
    dx, dw, db = ops.layer_norm_backward(dy, x, mean, rstd, w)
    d = dy.clone()
    dx2, dw2, db2 = ops.layer_norm_backward(d, x, mean, rstd, w, dx=d)
    assert same_bits(d, dx) and same_bits(dw, dw2) and same_bits(db, db2)


def test_layer_norm_large_offset_and_special_values():
    g = gen(13)
    x = randn(g, 12, 2048) + 1000.0                 # variance from the centred values, not E[x^2] - E[x]^2
    check_norm_forward(x, None, None)
    x = torch.full((3, 768), 5.0, device="cuda").to(BF16)
    check_norm_forward(x, None, None)                # no variance at all
    x = randn(g, 4, 768)
    x[1, 5], x[2, 700] = float("nan"), INF
    y, mean, rstd = ops.layer_norm_forward(x)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
    for r in (0, 3):                                 # the other rows are what they are alone
        assert same_bits(y[r:r + 1], ops.layer_norm_forward(x[r:r + 1])[0])


def norm_backward_reference(dy, x, mean, rstd, w):
    dy, x = dy.double(), x.double()
    r = rstd.double()[:, None]
    xh = (x - mean.double()[:, None]) * r
    gw = dy if w is None else dy * w.double()
    dx = r * (gw - gw.mean(1, keepdim=True) - xh * (gw * xh).mean(1, keepdim=True))
    size = r * (gw.abs() + gw.abs().mean(1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(1, keepdim=True))
    # x - mean rounds relative to x: that much of xhat is uncertain
    loose = r * (x.abs() + mean.double().abs()[:, None])
    size = size + r * (loose * (gw * xh).abs().mean(1, keepdim=True) + xh.abs() * (gw.abs() * loose).mean(1, keepdim=True))
    dw, dws = (dy * xh).sum(0), (dy.abs() * (xh.abs() + loose)).sum(0)
    return dx, size, dw, dws, dy.sum(0), dy.abs().sum(0)


def check_norm_backward(dy, x, mean, rstd, w, **kw):
    rows, cols = x.shape
    dx, dw, db = ops.layer_norm_backward(dy, x, mean, rstd, w, **kw)
    want, size, wdw, sdw, wdb, sdb = norm_backward_reference(dy, x, mean, rstd, w)
    close(dx, want, path(cols) * size, "dx")
    if dw is not None:
        close(dw, wdw, path(rows) * sdw, "dweight")
    if db is not None:
        close(db, wdb, path(rows) * sdb, "dbias")
    return dx, dw, db


@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("dtype,param", [(BF16, BF16), (FP16, FP32), (FP32, FP32), (BF16, FP32)])
def test_layer_norm_backward(rows, cols, dtype, param):
    g = gen(rows * 5 + cols)
    x = (randn(g, rows, cols) * 1.5 - 0.25).to(dtype)
    dy = (randn(g, rows, cols) * 0.1).to(dtype)
    w = (1 + 0.2 * randn(g, cols)).to(param)
    _, mean, rstd = ops.layer_norm_forward(x, w, None)
    a = check_norm_backward(dy, x, mean, rstd, w)
    b = ops.layer_norm_backward(dy, x, mean, rstd, w)
    assert all(same_bits(p, q) for p, q in zip(a, b))            # repeats bit for bit


@pytest.mark.parametrize("grad", [BF16, FP16, FP32])
@pytest.mark.parametrize("rows,cols", [(0, 768), (1, 768), (411, 768), (40, 1001)])
def test_layer_norm_weight_gradients_accumulate_into_an_arena(grad, rows, cols):
    """dweight and dbias in a gradient arena's type, written or added with one rounding."""
    g = gen(21)
    x, dy = randn(g, rows, cols).to(BF16), (randn(g, rows, cols) * 0.1).to(BF16)
    w = randn(g, cols).to(BF16)
    _, mean, rstd = ops.layer_norm_forward(x, w, None)
    arena = torch.full((2 * cols + 64,), 3.0, dtype=grad, device="cuda")
    dw, db = arena[16:16 + cols], arena[32 + cols:32 + 2 * cols]
    _, size, wdw, sdw, wdb, sdb = norm_backward_reference(dy, x, mean, rstd, w)
    ops.layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db)
    close(dw, wdw, path(rows) * sdw, "dweight")
    close(db, wdb, path(rows) * sdb, "dbias")
    dw.copy_(torch.linspace(-1, 1, cols, device="cuda"))
    old_w, old_b = dw.double(), db.double()
    ops.layer_norm_backward(dy, x, mean, rstd, w, dweight=dw, dbias=db, accumulate=True)
    close(dw, old_w + wdw, path(rows) * sdw + E * (old_w.abs() + wdw.abs()), "dweight added")
    close(db, old_b + wdb, path(rows) * sdb + E * (old_b.abs() + wdb.abs()), "dbias added")
    hole = torch.ones_like(arena, dtype=torch.bool)
    hole[16:16 + cols] = False
    hole[32 + cols:32 + 2 * cols] = False
    assert (arena[hole] == 3.0).all()
    # one of the two alone, and neither
    only = torch.empty(cols, dtype=grad, device="cuda")
    _, a, b = ops.layer_norm_backward(dy, x, mean, rstd, w, dweight=only, dbias=False)
    assert b is None
    close(only, wdw, path(rows) * sdw, "dweight alone")
    dx, a, b = ops.layer_norm_backward(dy, x, mean, rstd, w, dweight=False, dbias=False)
    assert a is None and b is None


def test_layer_norm_gradient_against_differences():
    """Central differences of sum(y * v) along a direction, in the kernel's own fp32
    forward pass: the rounding of y (E each, n values, random signs) over 2 h and
    the third derivative times h^2 are both below 1e-3 of the gradient's size here."""
    g = gen(31)
    x, v, d = randn(g, 6, 300), randn(g, 6, 300), randn(g, 6, 300)
    w, b = 1 + 0.2 * randn(g, 300), randn(g, 300)
    dw_dir = randn(g, 300)
    h = 2.0 ** -6
    y0, mean, rstd = ops.layer_norm_forward(x, w, b)
    f = lambda xx, ww, bb: (ops.layer_norm_forward(xx, ww, bb)[0].double() * v.double()).sum().item()  # noqa: E731
    dx, dw, db = ops.layer_norm_backward(v, x, mean, rstd, w)
    for grad, direction, plus, minus in (
            (dx, d, (x + h * d, w, b), (x - h * d, w, b)),
            (dw, dw_dir, (x, w + h * dw_dir, b), (x, w - h * dw_dir, b)),
            (db, dw_dir, (x, w, b + h * dw_dir), (x, w, b - h * dw_dir))):
        slope = (f(*plus) - f(*minus)) / (2 * h)
        want = (grad.double() * direction.double()).sum().item()
        size = grad.double().norm().item() * direction.double().norm().item()
        assert abs(slope - want) <= 1e-3 * size


# --------------------------------------------------------------------------
# embedding
# --------------------------------------------------------------------------

def check_embedding_forward(ids, table, scale, **kw):
    out = ops.embedding_forward(ids, table, scale, **kw)
    ok = (ids >= 0) & (ids < table.shape[0])
    want = table.double()[torch.where(ok, ids, torch.zeros_like(ids)).long()] * scale
    want = torch.where(ok[..., None], want, torch.zeros_like(want))
    close(out, want, 2 * E * want.abs(), "out")
    return out


@pytest.mark.parametrize("n,vocab,cols", [(0, 10, 8), (1, 1, 1), (1, 50257, 768), (5, 7, 33), (1000, 50257, 768),
                                          (4099, 1000, 513), (77, 300, 4096), (3, 20, 8200)])
@pytest.mark.parametrize("dtype,ids_dtype,scale", [(BF16, torch.int64, 1.0), (FP16, torch.int32, 27.712812921102035),
                                                   (FP32, torch.int64, 0.5)])
def test_embedding_forward(n, vocab, cols, dtype, ids_dtype, scale):
    g = gen(n + vocab + cols)
    table = (randn(g, vocab, cols) * 0.02).to(dtype)
    ids = torch.randint(vocab, (n,), generator=g, device="cuda").to(ids_dtype)
    check_embedding_forward(ids, table, scale)


def test_embedding_forward_bad_ids_strides_and_shapes():
    g = gen(41)
    table = strided(randn(g, 100, 96).to(BF16), 5, 3)
    ids = torch.randint(100, (4, 9), generator=g, device="cuda")
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert check_embedding_forward(ids, table, 2.0, bad_id=bad).shape == (4, 9, 96)
    assert bad.item() == 0
    ids[1, 2], ids[3, 3], ids[0, 0] = -1, 100, 2 ** 40
    table = table.clone()
    table[0, 0] = float("nan")                       # never read for a bad id
    ids[ids == 0] = 1
    check_embedding_forward(ids, table, 2.0, bad_id=bad)
    assert bad.item() == 1
    out = strided(torch.zeros(36, 96, dtype=BF16, device="cuda"), 11, 1)
    before = out._base.clone()
    check_embedding_forward(ids.flatten(), table, 1.0, out=out)
    assert gap_untouched(out, before)


def embedding_backward_reference(ids, dout, vocab, scale, padding_id=-1):
    cols = dout.shape[-1]
    ids, dout = ids.reshape(-1).long(), dout.reshape(-1, cols).double()
    keep = (ids >= 0) & (ids < vocab) & (ids != padding_id)
    want = torch.zeros(vocab, cols, dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(want), torch.zeros(vocab, 1, dtype=torch.float64, device="cuda")
    want.index_add_(0, ids[keep], dout[keep])
    size.index_add_(0, ids[keep], dout[keep].abs())
    count.index_add_(0, ids[keep], torch.ones(int(keep.sum()), 1, dtype=torch.float64, device="cuda"))
    return want * scale, size * abs(scale) * E * (count.clamp(max=512) + 64 + count / 256)


def check_embedding_backward(ids, dout, vocab, scale=1.0, grad=None, padding_id=-1, **kw):
    grad = dout.dtype if grad is None else grad
    dtable = torch.full((vocab, dout.shape[-1]), 9.0, dtype=grad, device="cuda")
    ops.embedding_backward(ids, dout, dtable, scale, padding_id=padding_id, **kw)
    want, slack = embedding_backward_reference(ids, dout, vocab, scale, padding_id)
    close(dtable, want, slack, "dtable")
    again = torch.full_like(dtable, -2.0)
    ops.embedding_backward(ids, dout, again, scale, padding_id=padding_id, **kw)
    assert same_bits(again, dtable)                  # repeats bit for bit
    return dtable


@pytest.mark.parametrize("n,vocab,cols", [(0, 10, 8), (1, 1, 1), (1, 50257, 768), (5, 7, 33), (31, 3, 40),
                                          (33, 33, 1), (1000, 50257, 768), (4099, 1000, 513), (8192, 50257, 64),
                                          (20000, 128256, 16), (3000, 200, 1024), (40000, 3, 72), (64, 300, 4104)])
@pytest.mark.parametrize("dtype,grad,ids_dtype", [(BF16, BF16, torch.int64), (FP16, FP32, torch.int32),
                                                  (FP32, FP32, torch.int64), (BF16, FP16, torch.int32)])
def test_embedding_backward(n, vocab, cols, dtype, grad, ids_dtype):
    g = gen(n + 3 * vocab + cols)
    ids = torch.randint(vocab, (n,), generator=g, device="cuda")
    ids = (ids * ids // max(vocab, 1)).to(ids_dtype)             # small ids more often
    dout = (randn(g, n, cols) * 0.05).to(dtype)
    check_embedding_backward(ids, dout, vocab, 1.0 if n % 2 else 8.0, grad)


@pytest.mark.parametrize("n", [1, 32, 33, 1024, 5000, 70001])
@pytest.mark.parametrize("cols", [8, 100])
def test_embedding_backward_of_one_token_repeated(n, cols):
    """Every token the same id: one long sum, split and joined."""
    g = gen(n)
    ids = torch.full((n,), 77, device="cuda")
    check_embedding_backward(ids, randn(g, n, cols), 500, 1.0)
    ids[n // 2:] = 78
    check_embedding_backward(ids, randn(g, n, cols).to(BF16), 500, 1.0, FP32)


def test_embedding_backward_many_ids_per_block():
    """A vocabulary with more ids than one block of the sort takes per SM."""
    g = gen(55)
    vocab = 400_003
    ids = torch.randint(vocab, (3000,), generator=g, device="cuda")
    ids[::7] = vocab - 1
    ids[1::7] = 0
    check_embedding_backward(ids, randn(g, 3000, 8), vocab, 1.0)


def test_embedding_backward_padding_bad_ids_strides_and_shapes():
    g = gen(56)
    ids = torch.randint(50, (6, 70), generator=g, device="cuda")
    dout = randn(g, 6, 70, 40).to(BF16)
    check_embedding_backward(ids, dout, 50, 1.5, FP32, padding_id=7)
    ids[0, 3], ids[5, 69], ids[2, 2] = -1, 50, 2 ** 40
    dout[0, 3], dout[5, 69] = float("nan"), INF      # tokens that take no part are not read
    check_embedding_backward(ids, dout, 50, 1.5, FP32, padding_id=7)
    every = torch.full((100,), 7, device="cuda")
    got = check_embedding_backward(every, torch.full((100, 24), float("nan"), device="cuda"), 50, 1.0, padding_id=7)
    assert (got == 0).all()
    d2 = strided(randn(g, 420, 40).to(BF16), 3, 1)
    table = strided(torch.zeros(50, 40, device="cuda"), 9, 2)
    before = table._base.clone()
    ops.embedding_backward(ids.flatten(), d2, table, 1.0)
    want, slack = embedding_backward_reference(ids, d2, 50, 1.0)
    close(table, want, slack, "strided")
    assert gap_untouched(table, before)
    one = randn(g, 1, 40).expand(420, 40)            # the gradient of a sum: one row for all
    check_embedding_backward(ids.flatten(), one, 50, 1.0)


@pytest.mark.parametrize("grad", [BF16, FP32])
@pytest.mark.parametrize("n,cols", [(0, 16), (300, 16), (5000, 99)])
def test_embedding_backward_adds_to_a_tied_heads_gradient(grad, n, cols):
    g = gen(57)
    vocab = 1000
    ids = torch.randint(40, (n,), generator=g, device="cuda") * 25
    dout = randn(g, n, cols).to(BF16)
    dtable = randn(g, vocab, cols).to(grad)
    dtable[1] = float("nan")                         # not an id of these tokens: stays as it is
    before = dtable.clone()
    ops.embedding_backward(ids, dout, dtable, 2.0, accumulate=True)
    want, slack = embedding_backward_reference(ids, dout, vocab, 2.0)
    used = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    used[ids] = True
    assert same_bits(dtable[~used], before[~used])
    close(dtable[used], (before.double() + want)[used],
          (slack + E * (before.double().abs() + want.abs()))[used], "added")


def test_embedding_backward_is_the_transpose_of_the_lookup():
    """<lookup(W + h D) - lookup(W - h D), V> / 2h = <D, gradient>, exactly linear: only rounding is left."""
    g = gen(58)
    ids = torch.randint(90, (700,), generator=g, device="cuda")
    table, d, v = randn(g, 90, 64), randn(g, 90, 64), randn(g, 700, 64)
    hi, lo = ops.embedding_forward(ids, table + d, 3.0), ops.embedding_forward(ids, table - d, 3.0)
    slope = ((hi.double() - lo.double()) * v.double()).sum().item() / 2
    dtable = torch.empty(90, 64, device="cuda")
    ops.embedding_backward(ids, v, dtable, 3.0)
    assert abs(slope - (dtable.double() * d.double()).sum().item()) <= 1e-5 * dtable.norm().item() * d.norm().item()


# --------------------------------------------------------------------------
# losses on logits
# --------------------------------------------------------------------------

def softmax_reference(z, temperature):
    """q, log q, and the distance from the maximum, of rows of logits."""
    z = z.double() / temperature
    top = z.amax(1, keepdim=True)
    d = z - top
    total = d.exp().sum(1, keepdim=True)
    logq = d - total.log()
    return logq.exp(), logq, torch.nan_to_num(d.abs(), nan=0.0, posinf=0.0)


def grad_slack(coef, q, target, dist, vocab):
    rel = path(vocab) + EXP * 2 + 4 * E * dist
    return coef.abs()[:, None] * (torch.nan_to_num(q) * rel + target * 64 * E)


def check_distill(logits, ids, teacher, weight=None, temperature=1.0, grad_scale=1.0, **kw):
    rows, vocab = logits.shape
    z0 = logits.clone()
    before = kw["grad"]._base.clone() if isinstance(kw.get("grad"), torch.Tensor) and kw["grad"]._base is not None else None
    loss, row, grad = ops.distill_loss(logits, ids, teacher, weight, temperature=temperature, grad_scale=grad_scale, **kw)
    w = torch.ones(rows, device="cuda").double() if weight is None else weight.double()
    ids, a = ids.long(), teacher.double() / temperature
    there = (ids >= 0) & (ids < vocab) & (a != -INF)
    a = torch.where(there, a, torch.full_like(a, -INF))
    on = (w != 0) & there.any(1)
    top = torch.where(on, a.amax(1), torch.zeros_like(w))[:, None]
    p = (a - top).exp()
    total = p.sum(1, keepdim=True)
    p, logp = p / total, a - top - total.log()
    q, logq, dist = softmax_reference(z0, temperature)
    at = torch.where(there, ids, torch.zeros_like(ids))
    terms = torch.where(p > 0, p * (logp - logq.gather(1, at)), torch.zeros_like(p))
    want = torch.where(on, temperature ** 2 * terms.sum(1), torch.zeros_like(w))
    p = torch.where(there & on[:, None], p, torch.zeros_like(p))
    err = path(vocab) + 2 * EXP + 8 * E * (dist.gather(1, at) + torch.nan_to_num((a - top).abs(), posinf=0.0))
    slack = temperature ** 2 * (p * (err + 64 * E * (1 + torch.nan_to_num(terms.abs() / p.clamp(min=1e-30), posinf=0.0)))).sum(1)
    close(row, want, slack, "row_loss")
    target = torch.zeros_like(q).scatter_add_(1, at, p)
    coef = grad_scale * w * temperature
    wgrad = torch.where(on[:, None], (q - target) * coef[:, None], torch.zeros_like(q))
    if grad is not None:
        close(grad, wgrad, grad_slack(coef, q, target, dist, vocab), "grad")
        if before is not None:
            assert gap_untouched(grad, before)
        assert (grad[~on] == 0).all()
    total_loss = torch.where(w != 0, w * want, torch.zeros_like(w))
    if torch.isfinite(total_loss).all():
        close(loss, total_loss.sum().reshape(1), (w.abs() * (slack + E * want.abs())).sum().item(), "loss")
    else:
        assert not torch.isfinite(loss).any()
    return loss, row, grad


def distill_inputs(seed, rows, vocab, k, dtype, spread=2.0):
    g = gen(seed)
    z = (randn(g, rows, vocab) * spread).to(dtype)
    ids = torch.argsort(torch.rand(rows, max(min(vocab, 4 * k), k), generator=g, device="cuda"), 1)[:, :k]
    ids = (ids * max(vocab // max(4 * k, 1), 1)) % vocab
    teacher = randn(g, rows, k) * 2 + 3
    return z, ids, teacher


LOGIT_SHAPES = [(1, 1), (1, 2), (3, 7), (2, 127), (5, 1000), (257, 999), (64, 4096), (33, 8191), (7, 32000),
                (200, 50257), (63, 50257), (3, 50304), (9, 128256), (1, 128256), (2, 131071), (300, 20011)]


@pytest.mark.parametrize("rows,vocab", LOGIT_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_distill_loss(rows, vocab, dtype):
    k = min(vocab, 16)
    z, ids, teacher = distill_inputs(rows + vocab, rows, vocab, k, dtype)
    weight = torch.rand(rows, generator=gen(3), device="cuda") / rows
    weight[1::3] = 0
    scale = 1024.0 if dtype == FP16 else 1.0
    check_distill(z, ids, teacher.to(dtype), weight, 1.0, scale)
    check_distill(z, ids.to(torch.int32), teacher, None, 2.5, scale / rows)


@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 64, 255, 256, 257, 500, 1000, 1024])
@pytest.mark.parametrize("vocab", [2048, 30001])
def test_distill_list_lengths(k, vocab):
    z, ids, teacher = distill_inputs(k, 9, vocab, k, BF16)
    check_distill(z, ids, teacher)


def test_distill_duplicate_empty_and_foreign_entries():
    z, ids, teacher = distill_inputs(71, 12, 5000, 40, FP32)
    ids[0, :20] = 4321                               # one id many times
    ids[1] = 17
    teacher[2, 5:] = -INF                            # a shorter list
    ids[2, 5:] = ids[2, 0:1]                         #   padded with an id that is in it
    ids[3, 10:] = -1
    ids[4, 1:] = 5000
    ids[5] = -100                                    # nothing left: the row counts as masked
    teacher[6] = -INF
    z[5, 3] = float("nan")
    z[6, 4] = INF
    ids[7, :] = torch.arange(40, device="cuda")      # first and last elements of the row
    ids[8, :] = 4999 - torch.arange(40, device="cuda")
    _, row, grad = check_distill(z, ids, teacher, None, 1.7)
    assert row[5] == 0 and row[6] == 0 and (grad[5] == 0).all() and (grad[6] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("vocab", [517, 50257])
def test_losses_with_masked_logits(dtype, vocab):
    """-inf and the type's lowest value in masked places; rows of nothing else."""
    z, ids, teacher = distill_inputs(81, 10, vocab, 8, dtype)
    low = torch.finfo(dtype).min
    z[0, ::2] = -INF
    z[1, 1::2] = low
    z[2] = low                                       # all equal: the uniform distribution
    z[3] = low
    z[3, 5] = 1.0
    z[4, : vocab - 1] = -INF                         # one element left
    ids[4] = vocab - 1
    z[5] = -INF                                      # nothing left: NaN
    z[6, 100] = float("nan")
    z[7, 100] = INF
    z[8, 3:] = -INF
    ids[8, :] = torch.arange(8, device="cuda") % 3
    ids[0] = 1 + 2 * torch.arange(8, device="cuda")
    ids[1] = 2 * torch.arange(8, device="cuda")
    ids[3] = 5
    loss, row, grad = check_distill(z, ids, teacher)
    assert torch.isnan(row[5:8]).all() and torch.isnan(grad[5:8]).all() and torch.isfinite(row[:5]).all()
    # a masked row hides all of it
    weight = torch.ones(10, device="cuda")
    weight[5:8] = 0
    loss, row, grad = check_distill(z, ids, teacher, weight)
    assert torch.isfinite(loss).all() and (grad[5:8] == 0).all()
    # a student that rules out what the teacher wants: infinite loss, finite gradient
    z[8, 2] = -INF
    loss, row, grad = check_distill(z, ids, teacher, weight)
    assert row[8] == INF and torch.isfinite(grad).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("pad,offset,gpad,goffset", [(47, 0, 47, 0), (0, 1, 0, 1), (3, 5, 3, 5), (8, 0, 16, 0),
                                                     (8, 0, 1, 1), (1, 3, 8, 0), (0, 0, 5, 2)])
@pytest.mark.parametrize("rows,vocab", [(5, 50257), (40, 1003), (3, 9), (2, 100000)])
def test_loss_strides_and_alignment(dtype, pad, offset, gpad, goffset, rows, vocab):
    z, ids, teacher = distill_inputs(91, rows, vocab, 5, dtype)
    z = strided(z, pad, offset)
    out = strided(torch.zeros(rows, vocab, dtype=dtype, device="cuda"), gpad, goffset)
    ids = strided(ids, 3, 1)
    teacher = strided(teacher, 2, 1)
    check_distill(z, ids, teacher, grad=out)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("rows,vocab,offset", [(11, 50257, 0), (700, 1003, 1), (3, 128256, 0), (2, 257, 3)])
def test_losses_in_place_and_alone(dtype, rows, vocab, offset):
    """The gradient over the logits; the loss without a gradient; the same bits every time."""
    z, ids, teacher = distill_inputs(92, rows, vocab, 6, dtype)
    z = strided(z, 2, offset)
    keep = z.clone()
    loss, row, grad = check_distill(z, ids, teacher)
    again = ops.distill_loss(z, ids, teacher)
    assert all(same_bits(a, b) for a, b in zip((loss, row, grad), again))
    alone = ops.distill_loss(z, ids, teacher, grad=False)
    assert alone[2] is None
    close(alone[1], row.double(), 2 * path(vocab) + 4 * EXP + E * 200, "row_loss alone")
    l2, r2, g2 = ops.distill_loss(z, ids, teacher, grad=z)
    assert g2 is z and same_bits(z, grad) and same_bits(r2, row)
    z.copy_(keep)
    tok, adv = ids[:, 0].contiguous(), randn(gen(4), rows)
    first = ops.policy_loss(z, tok, adv)
    assert same_bits(ops.policy_loss(z, tok, adv, grad=z)[3], first[3])


@pytest.mark.parametrize("dtype,vocab", [(FP32, 480_001), (BF16, 950_003), (FP16, 440_011)])
def test_losses_of_vocabularies_beyond_the_shared_memory_of_a_cluster(dtype, vocab):
    z, ids, teacher = distill_inputs(94, 3, vocab, 20, dtype)
    ids[1, 5] = ids[1, 4]
    weight = torch.tensor([0.5, 1.0, 0.0], device="cuda")
    check_distill(z, ids, teacher, weight, 1.5, 256.0 if dtype == FP16 else 1.0)
    zp, tokens, adv, old, ref = policy_inputs(95, 3, vocab, dtype)
    check_policy(zp, tokens, adv, weight, old, ref, kl=0.1, grad_scale=256.0 if dtype == FP16 else 1.0)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("at", [3, 700, 49_999])
def test_losses_of_rows_that_rise_far_above_their_first_elements(dtype, at):
    """One logit exceeds the others by far more than fp32's exponent holds (2^127 is 88 nats)."""
    z, ids, teacher = distill_inputs(96, 6, 50_257, 4, dtype)
    z[:, at] = torch.tensor([60.0, 88.0, 100.0, 300.0, 3e4, 1e30], device="cuda").to(dtype)
    ids[:, 0] = at
    check_distill(z, ids, teacher)
    check_policy(z, ids[:, 0].contiguous(), torch.ones(6, device="cuda"))
    z = -z.abs() * 40.0
    z[:, at] = 0.0
    check_distill(z, ids, teacher)


@pytest.mark.parametrize("rows,vocab,masked", [(1500, 20_011, 0.5), (3000, 300, 0.9), (700, 50_257, 0.0), (2000, 7, 0.3)])
def test_many_rows_with_masked_ones_among_them(rows, vocab, masked):
    z, ids, teacher = distill_inputs(97, rows, vocab, 3, BF16)
    weight = (torch.rand(rows, generator=gen(6), device="cuda") >= masked).float()
    check_distill(z, ids, teacher, weight)
    z[weight == 0] = float("nan")
    adv = randn(gen(7), rows)
    loss, row, logp, grad = check_policy(z, ids[:, 0].contiguous(), adv, weight)
    assert torch.isfinite(loss).all()


def test_distill_of_one_entry_is_cross_entropy():
    z, ids, _ = distill_inputs(93, 40, 3001, 1, FP32)
    loss, row, grad = check_distill(z, ids, torch.full((40, 1), -3.0, device="cuda"))
    want = -torch.log_softmax(z.double(), 1).gather(1, ids)[:, 0]
    assert (row.double() - want).abs().max() <= path(3001) + 4 * EXP + 64 * E * 10


def check_policy(logits, tokens, adv, weight=None, old=None, ref=None, temperature=1.0, low=0.2, high=0.2, kl=0.0,
                 grad_scale=1.0, **kw):
    rows, vocab = logits.shape
    z0 = logits.clone()
    loss, row, logp, grad = ops.policy_loss(logits, tokens, adv, weight, old_logp=old, ref_logp=ref,
                                            temperature=temperature, clip_low=low, clip_high=high, kl_coef=kl,
                                            grad_scale=grad_scale, **kw)
    w = torch.ones(rows, device="cuda").double() if weight is None else weight.double()
    tokens = tokens.long()
    on = (w != 0) & (tokens >= 0) & (tokens < vocab)
    at = torch.where(on, tokens, torch.zeros_like(tokens))[:, None]
    q, logq, dist = softmax_reference(z0, temperature)
    zero = torch.zeros_like(w)
    lp = torch.where(on, logq.gather(1, at)[:, 0], zero)        # a masked row's value and error are 0
    err = path(vocab) + 2 * EXP + 8 * E * (dist.gather(1, at)[:, 0] + lp.abs())
    close(logp, torch.where(on, lp, zero), err, "logp")
    a = adv.double()
    # the kink: rows within the error of logp of a clip bound may fall on either side
    r = (lp - (lp if old is None else old.double())).exp()
    re = r * (err + E * (8 + (0 if old is None else old.double().abs())) + EXP)
    free, held = r * a, r.clamp(1 - low, 1 + high) * a
    d = zero if ref is None else ref.double() - lp
    de = err + E * (0 if ref is None else ref.double().abs())
    want = torch.where(on, -torch.minimum(free, held) + kl * (torch.expm1(d) - d), zero)
    rslack = re * a.abs() + kl * (torch.expm1(d).abs() * de + de * de + 16 * E * (d.exp() + d.abs() + 1)) + 8 * E * want.abs()
    close(row, want, rslack, "row_loss")
    slope = -torch.where(held < free, zero, free) - kl * torch.expm1(d)
    sslack = re * a.abs() + kl * (d.exp() * (de + 16 * E)) + 8 * E * slope.abs()
    c = grad_scale * w / temperature
    rslack, sslack = torch.where(on, rslack, zero), torch.where(on, sslack, zero)
    q = torch.where(on[:, None], q, torch.zeros_like(q))
    target = torch.zeros_like(q).scatter_(1, at, 1.0)
    wgrad = torch.where(on[:, None], (target - q) * (c * slope)[:, None], torch.zeros_like(q))
    if grad is not None:
        slack = grad_slack(c * slope, q, target, dist, vocab) + (c * sslack).abs()[:, None] * (target - q).abs()
        close(grad, wgrad, slack, "grad")
        assert (grad[~on] == 0).all()
    close(loss, torch.where(on, w * want, zero).sum().reshape(1), (w.abs() * (rslack + E * want.abs())).sum().item(), "loss")
    return loss, row, logp, grad


def policy_inputs(seed, rows, vocab, dtype, temperature=1.0):
    g = gen(seed)
    z = (randn(g, rows, vocab) * 2).to(dtype)
    tokens = torch.randint(vocab, (rows,), generator=g, device="cuda")
    z.scatter_(1, tokens[:, None], (randn(g, rows, 1) + 6).to(dtype))
    lp = softmax_reference(z, temperature)[1].gather(1, tokens[:, None])[:, 0]
    d = 0.3 * randn(g, rows)
    for bound in (-math.log(0.8), -math.log(1.2), -math.log(1.28)):
        d = torch.where((d - bound).abs() < 1e-3, d + 2e-3, d)          # off the kinks
    return z, tokens, randn(g, rows), (lp + d).float(), (lp + 0.4 * randn(g, rows)).float()


@pytest.mark.parametrize("rows,vocab", LOGIT_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_policy_loss(rows, vocab, dtype):
    z, tokens, adv, old, ref = policy_inputs(rows + 2 * vocab, rows, vocab, dtype, 0.7)
    weight = torch.rand(rows, generator=gen(3), device="cuda") / rows
    weight[1::3] = 0
    scale = 1024.0 if dtype == FP16 else 1.0
    check_policy(z, tokens, adv, weight, old, ref, 0.7, 0.2, 0.28, 0.05, scale)
    check_policy(z, tokens.to(torch.int32), adv, None, None, None, 1.0, grad_scale=scale / rows)


def test_policy_clipping_and_masks():
    z, tokens, _, _, _ = policy_inputs(101, 16, 3000, FP32)
    lp = softmax_reference(z, 1.0)[1].gather(1, tokens[:, None])[:, 0].float()
    adv = torch.tensor([1.0, -1.0] * 8, device="cuda")
    shift = torch.tensor([0.5, 0.5, -0.5, -0.5, 0.1, 0.1, -0.1, -0.1] * 2, device="cuda")
    old = lp - shift                                  # ratio exp(shift)
    _, _, _, grad = check_policy(z, tokens, adv, None, old, None)
    gone = (grad == 0).all(1).tolist()
    # clipped: the ratio above with a gain, or below with a loss
    assert gone == [True, False, False, True, False, False, False, False] * 2
    check_policy(z, tokens, adv, None, old, None, low=1.0, high=INF)     # no bounds at all
    check_policy(z, tokens, adv, None, old, lp + 2.0, kl=0.5)            # far from the reference
    check_policy(z, tokens, torch.zeros(16, device="cuda"), None, old, None)
    tokens[0], tokens[1], tokens[2] = -100, 3000, 2 ** 40                # outside the vocabulary: masked
    weight = torch.ones(16, device="cuda")
    weight[3] = 0
    z[0, 5], z[3, 7] = float("nan"), INF
    loss, row, logp, grad = check_policy(z, tokens, adv, weight, old, None)
    assert torch.isfinite(loss).all() and (logp[:4] == 0).all()
    z[4] = -INF                                                          # a row of nothing: NaN
    row = ops.policy_loss(z, tokens, adv, weight, old_logp=old)
    assert torch.isnan(row[1][4]) and torch.isnan(row[3][4]).all() and torch.isnan(row[0]).all()
    none = torch.zeros(16, device="cuda")
    loss, row, logp, grad = check_policy(z, tokens, adv, none, old, None)
    assert loss.item() == 0 and (grad == 0).all()


@pytest.mark.parametrize("which", ["distill", "policy"])
def test_losses_of_no_rows(which):
    z = torch.empty(0, 100, device="cuda")
    loss = torch.full((1,), 5.0, device="cuda")
    if which == "distill":
        ops.distill_loss(z, torch.empty(0, 4, dtype=torch.int64, device="cuda"), torch.empty(0, 4, device="cuda"), loss=loss)
    else:
        ops.policy_loss(z, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), loss=loss)
    assert loss.item() == 0


@pytest.mark.parametrize("which", ["distill", "policy"])
def test_loss_gradients_against_differences(which):
    """Central differences along a direction of the kernel's own fp32 loss: rounding
    (path + EXP of a loss of a few units) over 2 h and the third derivative times
    h^2 stay below 2e-3 of |gradient| |direction|."""
    z, ids, teacher = distill_inputs(111, 8, 600, 12, FP32, 1.0)
    direction = (ops.distill_loss(z, ids, teacher)[2] * 8).contiguous()
    direction = direction / direction.norm()
    adv, ref = randn(gen(1), 8) + 2.0, torch.full((8,), -4.0, device="cuda")
    old = ops.policy_loss(z, ids[:, 0].contiguous(), adv)[2] + 0.05

    def f(zz):
        if which == "distill":
            return ops.distill_loss(zz, ids, teacher, temperature=1.3)
        r = ops.policy_loss(zz, ids[:, 0].contiguous(), adv, old_logp=old, ref_logp=ref, kl_coef=0.1)
        return r[0], r[1], r[3]

    h = 2.0 ** -5
    grad = f(z)[2].double()
    slope = (f(z + h * direction)[1].double() - f(z - h * direction)[1].double()).sum().item() / (2 * h)
    want = (grad * direction.double()).sum().item()
    assert abs(slope - want) <= 2e-3 * grad.norm().item()


def test_operators_on_a_side_stream_and_in_a_graph():
    z, ids, teacher = distill_inputs(121, 20, 50257, 8, BF16)
    tokens, adv = ids[:, 0].contiguous(), randn(gen(2), 20)
    table = randn(gen(3), 50257, 64)
    want = ops.distill_loss(z, ids, teacher), ops.policy_loss(z, tokens, adv), ops.embedding_forward(tokens, table)
    dtable = torch.empty_like(table)
    ops.embedding_backward(tokens, want[2], dtable)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = ops.distill_loss(z, ids, teacher, stream=side)
    b = ops.policy_loss(z, tokens, adv, stream=side)
    d2 = torch.empty_like(table)
    side.wait_stream(torch.cuda.current_stream())
    ops.embedding_backward(tokens, want[2], d2, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same_bits(p, q) for p, q in zip(a + b + (d2,), want[0] + want[1] + (dtable,)))
    graph = torch.cuda.CUDAGraph()
    x = randn(gen(5), 20, 64)
    with torch.cuda.graph(graph):
        ga = ops.distill_loss(z, ids, teacher)
        gb = ops.policy_loss(z, tokens, adv)
        ops.embedding_backward(tokens, want[2], d2)
        y, mean, rstd = ops.layer_norm_forward(x)
        dn = ops.layer_norm_backward(x, x, mean, rstd)
    d2.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(same_bits(p, q) for p, q in zip(ga + gb + (d2,), want[0] + want[1] + (dtable,)))
    assert same_bits(y, ops.layer_norm_forward(x)[0])
    assert all(same_bits(p, q) for p, q in zip(dn, ops.layer_norm_backward(x, x, mean, rstd)))


def test_refusals_on_tensors():
    x = torch.zeros(4, 64, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    stats = torch.zeros(4, device="cuda")
    calls = [
        lambda: ops.layer_norm_forward(x.double()),
        lambda: ops.layer_norm_forward(x.cpu()),
        lambda: ops.layer_norm_forward(x.t()),
        lambda: ops.layer_norm_forward(x, x[0, :63].contiguous()),
        lambda: ops.layer_norm_forward(x, x[0].to(BF16)),
        lambda: ops.layer_norm_forward(x, eps=-1.0),
        lambda: ops.layer_norm_forward(x, eps=float("nan")),
        lambda: ops.layer_norm_forward(x, out=x[:3]),
        lambda: ops.layer_norm_forward(x, save_stats=False, mean=stats),
        lambda: ops.layer_norm_forward(x[:, :0]),
        lambda: ops.layer_norm_backward(x, x[:2], stats, stats),
        lambda: ops.layer_norm_backward(x, x, stats, None),
        lambda: ops.layer_norm_backward(x, x, stats, stats, accumulate=True),
        lambda: ops.layer_norm_backward(x, x, stats, stats, scratch=torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: ops.embedding_forward(ids.float(), x),
        lambda: ops.embedding_forward(ids, x, float("inf")),
        lambda: ops.embedding_forward(ids, x[0]),
        lambda: ops.embedding_backward(ids, x[:3], x.clone()),
        lambda: ops.embedding_backward(ids, x, x.clone().t()),
        lambda: ops.embedding_backward(ids, x, x.clone(), scratch=torch.empty(8, dtype=torch.uint8, device="cuda")),
        lambda: ops.distill_loss(x, ids[:, None], x[:, :1], temperature=0.0),
        lambda: ops.distill_loss(x, ids[:, None], x[:, :2]),
        lambda: ops.distill_loss(x, ids[:, None].expand(4, 1025), x[:, :1].expand(4, 1025)),
        lambda: ops.distill_loss(x, ids[:, None], x[:, :1], grad_scale=float("nan")),
        lambda: ops.distill_loss(x, ids[:, None], x[:, :1], weight=ids),
        lambda: ops.policy_loss(x, ids, stats, kl_coef=0.1),
        lambda: ops.policy_loss(x, ids, stats, clip_low=1.5),
        lambda: ops.policy_loss(x, ids, stats, clip_high=-0.1),
        lambda: ops.policy_loss(x, ids[:3], stats),
        lambda: ops.policy_loss(x, ids, stats, grad=x.to(BF16)),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(B.SuperOffloadError) as err:
            call()
        assert err.value.status == B.SO_ERR_INVALID_ARG, i
    assert (x == 0).all()

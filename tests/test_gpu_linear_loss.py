"""Cross entropy from the hidden states against the formulas in 64 bits.

Tolerances.  u(T) is half a step of a type relative to a value (2^-8 bf16, 2^-11
fp16, 2^-24 fp32).  Logits: products of 16-bit numbers are exact in fp32; sums of d of
them on the tensor cores are taken to lose at most 2^-22 of the sum of magnitudes at
each of d / 16 + 8 additions (they may truncate), so with A = |h| |w| summed,
dz = (d / 16 + 8) 2^-22 A.  A row's loss is off by 2 max dz, the exponentials' 2^-21,
and 2^-22 of the numbers it is the difference of.  P is off by (2 max dz + 2^-20) of
|w| (q + [label]) from all that, and by u of its parts from its rounding: u(T), or
2^-21 for the several parts behind an fp32 gradient (fp16: 11 + 11 bits); in fp16 it is
held in multiples of 2^-39 of twice the largest weight.  The gradients' sums add
(n / 16 + 8) 2^-22 of their terms' magnitudes, splits and pieces 64 further roundings
of 2^-24, and one rounding of the result."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_operators import BF16, FP16, FP32, U, close, gap_untouched, gen, randn, same_bits, strided

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def reference(hidden, table, labels, weight, grad_scale):
    """(loss, row_loss, dhidden, dtable) and the slack of each, in 64 bits."""
    vocab, d = table.shape
    live = (labels >= 0) & (labels < vocab)
    if weight is not None:
        live &= weight != 0
    index = live.nonzero()[:, 0]
    h, w = hidden[index].double(), table.double()
    wt = torch.ones(index.numel(), device="cuda", dtype=torch.float64) if weight is None else weight[index].double()
    at = labels[index].long()[:, None]
    z = h @ w.t()
    dz = (d / 16 + 8) * 2.0 ** -22 * (h.abs() @ w.abs().t()).amax(1) if index.numel() else z.sum(1)
    lse = torch.logsumexp(z, 1)
    zl = z.gather(1, at)[:, 0]
    row = torch.zeros(hidden.shape[0], dtype=torch.float64, device="cuda")
    row_slack = torch.zeros_like(row)
    row[index] = lse - zl
    row_slack[index] = 2 * dz + 2.0 ** -21 + 2.0 ** -22 * (z.abs().amax(1) + lse.abs()) if index.numel() else 0.0
    q = torch.softmax(z, 1)
    one = torch.zeros_like(q).scatter_(1, at, 1.0)
    p = wt[:, None] * (q - one)
    unit = 2.0 ** -38 * (wt.abs().max() if index.numel() else 0.0) if hidden.dtype == FP16 else 0.0
    first = wt.abs()[:, None] * (q + one) * (2 * dz + 2.0 ** -20)[:, None] + unit
    s = grad_scale
    dh = torch.zeros(hidden.shape, dtype=torch.float64, device="cuda")
    dh_slack = torch.zeros_like(dh)
    dh[index] = s * (p @ w)
    dh_slack[index] = abs(s) * ((first + (U[hidden.dtype] + (vocab / 16 + 72) * 2.0 ** -22) * p.abs()) @ w.abs())
    dt = s * (p.t() @ h)

    def dt_slack(parts):
        return abs(s) * ((first + (parts + (index.numel() / 16 + 72) * 2.0 ** -22) * p.abs()).t() @ h.abs())

    full = torch.ones_like(row) if weight is None else weight.double()
    full = torch.where(live, full, torch.zeros_like(full))
    loss = (full * row).sum()
    loss_slack = (full.abs() * row_slack).sum() + 2.0 ** -22 * (full * row).abs().sum()
    return (loss, row, dh, dt), (loss_slack, row_slack, dh_slack, dt_slack)


def check(hidden, table, labels, weight=None, grad_scale=1.0, out=None, **kw):
    if out is not None and "dtable" not in kw:
        kw["dtable"] = torch.empty(table.shape, dtype=out, device="cuda")
    before = kw["dtable"].double() if kw.get("accumulate") else 0.0
    want, slack = reference(hidden, table, labels, weight, grad_scale)
    got = ops.linear_cross_entropy(hidden, table, labels, weight, grad_scale=grad_scale, **kw)
    close(got[0][0], want[0], slack[0], "loss")
    close(got[1], want[1], slack[1], "row_loss")
    if got[2] is not None:
        close(got[2], want[2], slack[2], "dhidden")
    if got[3] is not None:
        parts = 2.0 ** -21 if got[3].dtype == FP32 else U[hidden.dtype]
        close(got[3], before + want[3], slack[3](parts) + (0 if isinstance(before, float) else 2.0 ** -23 * before.abs()), "dtable")
    return got


def inputs(seed, rows, vocab, cols, dtype, ids=torch.int64, sharp=2.0):
    g = gen(seed)
    hidden, table = randn(g, rows, cols).to(dtype), (randn(g, vocab, cols) * sharp * cols ** -0.5).to(dtype)
    labels = torch.randint(vocab, (rows,), generator=g, device="cuda", dtype=ids)
    return g, hidden, table, labels


SHAPES = [(1, 1, 1), (1, 1000, 64), (3, 7, 8), (63, 257, 100), (128, 256, 64), (64, 3001, 768), (129, 255, 65), (200, 4097, 256),
          (256, 512, 1001), (257, 1000, 257), (600, 2000, 520), (1000, 777, 63), (31, 50257, 96)]


@pytest.mark.parametrize("rows,vocab,cols", SHAPES)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (FP16, FP32), (BF16, FP32), (FP16, BF16)])
def test_loss_and_gradients(rows, vocab, cols, dtype, out):
    _, hidden, table, labels = inputs(rows + vocab + cols, rows, vocab, cols, dtype, torch.int32 if rows % 2 else torch.int64)
    check(hidden, table, labels, out=out)


@pytest.mark.parametrize("rows,vocab,cols", [(1, 50257, 768), (300, 9000, 128)])
def test_what_is_left_out_is_not_computed(rows, vocab, cols):
    _, hidden, table, labels = inputs(5, rows, vocab, cols, BF16)
    whole = check(hidden, table, labels)
    for kw in (dict(dhidden=False), dict(dtable=False), dict(dhidden=False, dtable=False)):
        got = ops.linear_cross_entropy(hidden, table, labels, **kw)
        for name, a, b in zip(("loss", "row_loss", "dhidden", "dtable"), got, whole):
            if name in kw:
                assert a is None
            else:
                assert same_bits(a, b)


@pytest.mark.parametrize("rows", [40, 700])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (FP16, FP32)])
def test_masked_rows_are_not_read(rows, dtype, out):
    g, hidden, table, labels = inputs(6, rows, 1500, 200, dtype)
    weight = torch.rand(rows, generator=g, device="cuda") * (torch.rand(rows, generator=g, device="cuda") < 0.6) / rows
    labels[::7] = -100
    labels[3::11] = 1500
    gone = (weight == 0) | (labels < 0) | (labels >= 1500)
    assert 0 < gone.sum() < rows
    hidden[gone] = NAN
    hidden[gone.nonzero()[0]] = INF
    scale = 65536.0 if dtype == FP16 else 1.0
    got = check(hidden, table, labels, weight, grad_scale=scale, out=out)
    assert (got[1][gone] == 0).all() and (got[2][gone] == 0).all()


@pytest.mark.parametrize("rows", [0, 5, 200])
def test_no_row_takes_part(rows):
    hidden = torch.full((rows, 72), NAN, dtype=BF16, device="cuda")
    table = randn(gen(1), 300, 72).to(BF16)
    labels = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    loss, row, dh, dt = ops.linear_cross_entropy(hidden, table, labels)
    assert loss.item() == 0 and (row == 0).all() and (dh == 0).all() and (dt == 0).all() and dt.shape == (300, 72)
    kept = randn(gen(2), 300, 72)
    dt = kept.clone()
    ops.linear_cross_entropy(hidden, table, labels, dtable=dt, accumulate=True)
    assert torch.equal(dt, kept)


@pytest.mark.parametrize("pad,offset", [(8, 0), (8, 8), (1, 0), (3, 5)])
@pytest.mark.parametrize("cols", [96, 77])
def test_strides_and_alignment(pad, offset, cols):
    g, hidden, table, labels = inputs(7, 150, 5000, cols, BF16)
    h, t = strided(hidden, pad, offset), strided(table, pad, offset)
    dh = strided(torch.zeros_like(hidden), pad + 2, offset)
    for out in (BF16, FP32):
        dt = strided(torch.zeros(table.shape, dtype=out, device="cuda"), pad + 1, offset)
        before = [x._base.clone() for x in (dh, dt)]
        got = check(h, t, labels, dhidden=dh, dtable=dt)
        assert all(gap_untouched(x, b) for x, b in zip((dh, dt), before))
        plain = ops.linear_cross_entropy(hidden, table, labels, dtable=torch.empty_like(dt, memory_format=torch.contiguous_format))
        assert all(same_bits(a, b) for a, b in zip(got, plain))


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("rows", [60, 300])
def test_accumulates(dtype, rows):
    g, hidden, table, labels = inputs(8, rows, 1000, 136, BF16)
    check(hidden, table, labels, dtable=randn(g, 1000, 136).to(dtype), accumulate=True, grad_scale=0.25)
    check(hidden, table, labels, dtable=randn(g, 1000, 137).to(dtype)[:, 1:], accumulate=True)


def test_in_place_broadcast_rows_streams_and_scratch():
    g, hidden, table, labels = inputs(9, 300, 2000, 128, BF16)
    want = ops.linear_cross_entropy(hidden, table, labels)
    h = hidden.clone()
    got = ops.linear_cross_entropy(h, table, labels, dhidden=h)
    assert all(same_bits(a, b) for a, b in zip(got, want)) and got[2] is h
    check(hidden[:1].expand(300, 128), table, labels)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.linear_cross_entropy(hidden, table, labels, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(same_bits(a, b) for a, b in zip(got, want))
    need = B.so_linear_cross_entropy_scratch(300, 2000, 128, B.SO_DTYPE_BF16, B.SO_DTYPE_BF16, 1, 0)
    room = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN in every type
    got = ops.linear_cross_entropy(hidden, table, labels, scratch=room)
    assert all(same_bits(a, b) for a, b in zip(got, want))


def test_many_rows_in_several_pieces():
    g, hidden, table, labels = inputs(10, 17000, 9001, 72, BF16)
    weight = (torch.rand(17000, generator=g, device="cuda") < 0.8).float() / 17000
    check(hidden, table, labels, weight, out=FP32)


def test_special_values():
    g, hidden, table, labels = inputs(11, 200, 600, 64, BF16)
    hidden[5, 3] = NAN
    loss, row, dh, dt = ops.linear_cross_entropy(hidden, table, labels)
    bad = torch.zeros(200, dtype=torch.bool, device="cuda")
    bad[5] = True
    assert torch.isnan(loss).all() and torch.equal(torch.isnan(row), bad)
    assert torch.equal(torch.isnan(dh).all(1), bad) and torch.equal(torch.isnan(dh).any(1), bad) and torch.isnan(dt).all()
    # whole tiles of logits at -inf have no probability
    _, hidden, table, labels = inputs(12, 150, 1100, 64, BF16)
    hidden[:, 0] = 1.0
    table[256:900, 0] = -INF
    labels = labels % 256
    kept = torch.cat([table[:256], table[900:]])
    got = ops.linear_cross_entropy(hidden, table, labels, dhidden=False)
    want, slack = reference(hidden, kept, labels, None, 1.0)
    close(got[1], want[1], slack[1], "row_loss")
    assert (got[3][256:900] == 0).all()
    # one logit far above the others: the loss of its label is next to nothing, and no NaN comes of it
    _, hidden, table, labels = inputs(13, 150, 700, 64, FP16, sharp=100.0)
    check(hidden, table, labels)


def test_gradient_against_differences():
    """Central differences of the loss in one direction: the third derivative leaves (step^2 / 6) of
    a number of order 1, and the two losses are off by their slack."""
    g, hidden, table, labels = inputs(14, 96, 500, 64, BF16)
    weight = torch.rand(96, generator=g, device="cuda") / 96
    _, _, dh, dt = ops.linear_cross_entropy(hidden, table, labels, weight, dtable=torch.empty(500, 64, device="cuda"))
    for which, grad in ((0, dh), (1, dt)):
        at = (hidden, table)[which]
        way = (randn(g, *at.shape) * (2.0 ** -4 if which == 0 else 2.0 ** -6)).to(BF16)
        sides = []
        for sign in (1.0, -1.0):
            moved = [hidden, table]
            moved[which] = (at.float() + sign * way.float()).to(BF16)
            sides.append((moved[which], reference(*moved, labels, weight, 1.0)[0][0]))
        # the points as rounded; around their middle
        step = sides[0][0].double() - sides[1][0].double()
        middle = [hidden, table]
        middle[which] = ((sides[0][0].double() + sides[1][0].double()) / 2).to(BF16)
        _, _, mh, mt = ops.linear_cross_entropy(*middle, labels, weight, dtable=torch.empty(500, 64, device="cuda"))
        along = ((mh, mt)[which].double() * step).sum()
        size = ((mh, mt)[which].double().abs() * step.abs()).sum()
        assert (along - (sides[0][1] - sides[1][1])).abs() <= 0.02 * size


def test_captured_and_replayed():
    g, hidden, table, labels = inputs(15, 260, 3000, 160, BF16)
    out = ops.linear_cross_entropy(hidden, table, labels)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ops.linear_cross_entropy(hidden, table, labels, loss=out[0], row_loss=out[1], dhidden=out[2], dtable=out[3])
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(2):
        hidden.copy_(randn(g, 260, 160))
        labels.copy_(torch.randint(-300, 3000, (260,), generator=g, device="cuda"))
        graph.replay()
        got = [t.clone() for t in out]
        assert all(same_bits(a, b) for a, b in zip(got, ops.linear_cross_entropy(hidden, table, labels)))


class no_patience:
    def __init__(self, unit=-1):
        self.unit = unit

    def __enter__(self):
        B.so_debug_set_operator_polls(0, self.unit)

    def __exit__(self, *_):
        B.so_debug_set_operator_polls(1 << 20)


@pytest.mark.parametrize("rows", [50, 600])
def test_waits_that_run_out_make_everything_nan(rows):
    g, hidden, table, labels = inputs(16, rows, 9000, 200, BF16)
    want = ops.linear_cross_entropy(hidden, table, labels)
    for unit in (-1, 0):
        with no_patience(unit):
            got = ops.linear_cross_entropy(hidden, table, labels)
            alone = ops.linear_cross_entropy(hidden, table, labels, dhidden=False, dtable=False)
        assert all(torch.isnan(t).all() for t in (*got, *alone[:2]))
    assert all(same_bits(a, b) for a, b in zip(ops.linear_cross_entropy(hidden, table, labels), want))

"""What the operators' kernels leave behind when a wait of theirs runs out: NaN in every
result that depends on it, the others as ever, nothing in flight.  The limit is set to
zero, in one block (or cluster) of a launch or in all of them, so that they give up
without a look; the waits that drain copies keep their full limit."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_operators import BF16, FP16, FP32, gen, randn, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


class no_patience:
    def __init__(self, unit=-1):
        self.unit = unit

    def __enter__(self):
        B.so_debug_set_operator_polls(0, self.unit)

    def __exit__(self, *_):
        B.so_debug_set_operator_polls(1 << 20)


def rows_gone(got, want):
    """Which rows are NaN throughout; the others are what they should be, bit for bit."""
    gone = torch.isnan(got).reshape(got.shape[0], -1).all(1)
    assert same_bits(got[~gone], want[~gone])
    return gone


# aligned rows (one, several groups of threads to a block; several warps a row), odd ones
NORM_WIDTHS = [(5000, 256, BF16), (3001, 768, FP16), (2000, 4096, BF16), (900, 4096, FP32), (3000, 515, BF16), (1200, 6001, FP16),
               (2000, 101, FP32)]


@pytest.mark.parametrize("rows,cols,dtype", NORM_WIDTHS)
def test_layer_norm_rows_whose_copies_do_not_arrive(rows, cols, dtype):
    g = gen(rows + cols)
    x, dy = randn(g, rows, cols).to(dtype), randn(g, rows, cols).to(dtype)
    w, b = randn(g, cols), randn(g, cols)
    want = ops.layer_norm_forward(x, w, b)
    back = ops.layer_norm_backward(dy, x, want[1], want[2], w)
    for unit in (-1, 0, 3):
        with no_patience(unit):
            y, mean, rstd = ops.layer_norm_forward(x, w, b)
            dx, dw, db = ops.layer_norm_backward(dy, x, want[1], want[2], w)
        gone = rows_gone(y, want[0])
        assert torch.equal(rows_gone(mean[:, None], want[1][:, None]), gone)
        assert torch.equal(rows_gone(rstd[:, None], want[2][:, None]), gone)
        assert gone.all() if unit < 0 else 0 < gone.sum() < rows
        gone = rows_gone(dx, back[0])
        assert gone.all() if unit < 0 else 0 < gone.sum() < rows
        assert torch.isnan(dw).all() and torch.isnan(db).all()
    # in place as well: no row is left as it was
    z, d = x.clone(), dy.clone()
    with no_patience():
        ops.layer_norm_forward(z, w, b, out=z)
        ops.layer_norm_backward(d, x, want[1], want[2], w, dx=d)
    assert torch.isnan(z).all() and torch.isnan(d).all()
    again = ops.layer_norm_forward(x, w, b) + ops.layer_norm_backward(dy, x, want[1], want[2], w)
    assert all(same_bits(p, q) for p, q in zip(again, want + back))


# one block a row, two, eight; balanced and not; the loss alone
LOSS_SHAPES = [(700, 50_257, BF16), (400, 128_256, BF16), (20, 128_256, FP16), (300, 20_011, FP32), (9, 50_257, FP32)]


def loss_calls(rows, vocab, dtype):
    g = gen(rows + vocab)
    z = (randn(g, rows, vocab) * 2).to(dtype)
    ids = torch.randint(vocab, (rows, 6), generator=g, device="cuda")
    teacher, adv = randn(g, rows, 6), randn(g, rows)
    weight = (torch.rand(rows, generator=g, device="cuda") < 0.6).float()
    weight[0] = 0.0
    return z, weight, {
        "distill": lambda zz, w, grad: ops.distill_loss(zz, ids, teacher, w, grad=grad),
        "policy": lambda zz, w, grad: ops.policy_loss(zz, ids[:, 0].contiguous(), adv, w, grad=grad)}


@pytest.mark.parametrize("rows,vocab,dtype", LOSS_SHAPES)
@pytest.mark.parametrize("which", ["distill", "policy"])
def test_losses_whose_waits_run_out(rows, vocab, dtype, which):
    z, weight, calls = loss_calls(rows, vocab, dtype)
    fn = calls[which]
    want = fn(z, weight, None)
    alone = fn(z, weight, False)
    for unit in (-1, 0, 5):
        with no_patience(unit):
            got = fn(z, weight, None)
            only = fn(z, weight, False)
        gone = rows_gone(got[-1], want[-1])              # whole rows of the gradient, masked ones too
        assert gone.all() if unit < 0 else 0 < gone.sum() < rows
        per_row = torch.stack(got[1:-1], 1)
        assert torch.equal(rows_gone(per_row, torch.stack(want[1:-1], 1)), gone)
        gone_alone = rows_gone(torch.stack(only[1:-1], 1), torch.stack(alone[1:-1], 1))
        assert gone_alone.all() if unit < 0 else 0 < gone_alone.sum() < rows
        for g, w, lost in ((got, want, gone), (only, alone, gone_alone)):
            if (lost & (weight != 0)).any():
                assert torch.isnan(g[0]).all()
            else:
                assert same_bits(g[0], w[0])
    # over the logits: none of them is left in the place of a gradient
    zz = z.clone()
    with no_patience():
        fn(zz, weight, zz)
    assert torch.isnan(zz).all()
    assert all(same_bits(p, q) for p, q in zip(fn(z, weight, None), want))

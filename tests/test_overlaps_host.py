"""Outputs that lie partly in other tensors of a call are refused, ones that lie between their
rows are not: decided from addresses, sizes and strides before anything is launched."""
from __future__ import annotations

import pytest

from paper_2509_21271_b200 import binding as B
from test_more_operators_host import BACKWARD, FORWARD, LINEAR, _built  # noqa: F401
from test_operators_host import A, BF16, FP32, refused

F = dict(FORWARD, x=A, block=2 * A, h=3 * A, y=4 * A, gate=5 * A, post_weight=6 * A, post_bias=7 * A, weight=8 * A,
         bias=9 * A, stats=10 * A, rows=6, cols=96, x_stride=200, block_stride=200, h_stride=200, y_stride=200)   # fp16
ROW = 200 * 2                                             # bytes from a row to the next


def refuses(fn, good, **change):
    return refused(fn, *dict(good, **change).values())


@pytest.mark.parametrize("out,other", [("h", "x"), ("h", "block"), ("h", "y"), ("y", "x"), ("y", "block"), ("y", "h")])
@pytest.mark.parametrize("shift", [ROW, -ROW, 5 * ROW, -5 * ROW, 2, -2, 190, -190, ROW + 190, 2 * ROW - 190])
def test_residual_norm_forward_shifted(out, other, shift):
    """A row further, an element further, over a row's last elements or its first."""
    assert refuses(B.so_residual_norm_forward, F, **{out: F[other] + shift})


def test_residual_norm_forward_other_strides():
    """x's rows are 200 apart and y's 300: y's second row begins in x's, or in the gap behind it."""
    inside = 3 * ROW - 300 * 2 + 100
    assert refuses(B.so_residual_norm_forward, F, y=F["x"] + inside, y_stride=300)
    assert refuses(B.so_residual_norm_forward, F, x_stride=0, y=F["x"] - 3 * ROW)       # one row for all


G = dict(BACKWARD, dy=A, dh=2 * A, h=3 * A, block=4 * A, stats=5 * A, gate=6 * A, post_weight=7 * A, post_bias=8 * A, weight=9 * A,
         dx=10 * A, dblock=11 * A, dgate=12 * A, dpost_weight=13 * A, dpost_bias=14 * A, dweight=15 * A, dbias=16 * A, scratch=32 * A,
         rows=6, cols=96, dy_stride=200, dh_stride=200, h_stride=200, block_stride=200, dx_stride=200, dblock_stride=200)


@pytest.mark.parametrize("out", ["dx", "dblock"])
@pytest.mark.parametrize("other", ["dy", "dh", "h", "block", "dx", "dblock"])
@pytest.mark.parametrize("shift", [ROW, -ROW, 2, 190, -190])
def test_residual_norm_backward_shifted(out, other, shift):
    if out != other:
        assert refuses(B.so_residual_norm_backward, G, **{out: G[other] + shift})


L = dict(LINEAR, hidden=A, table=2 * A, labels=3 * A, weight=4 * A, dhidden=5 * A, dtable=6 * A, row_loss=7 * A, loss=8 * A,
         scratch=9 * A, rows=5, vocab=100, cols=64, hidden_stride=128, table_stride=128, dhidden_stride=128, dtable_stride=128,
         dtype=BF16, grad_dtype=FP32)


@pytest.mark.parametrize("out,other,shift", [
    ("dhidden", "hidden", 256), ("dhidden", "hidden", -256), ("dhidden", "hidden", 2), ("dhidden", "hidden", -126),
    ("dhidden", "table", 256 * 99 + 126), ("dtable", "table", 4), ("dtable", "hidden", 252), ("dtable", "dhidden", 4),
    ("dtable", "table", -512 * 99 - 252), ("dtable", "hidden", -512 * 50), ("dhidden", "dtable", 512 * 99 + 254)])
def test_linear_cross_entropy_shifted(out, other, shift):
    assert refuses(B.so_linear_cross_entropy, L, **{out: L[other] + shift})

"""Matrices of one row, whose row stride says nothing: a row of a wider buffer in place, and
strides that no matrix of more rows could have."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_linear_loss import check, inputs
from test_gpu_operators import BF16, FP32, gen, randn, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def last_token(t, length=7):
    """The same row as the last one of a sequence: shape [1, cols], stride length * cols."""
    buf = torch.zeros(1, length, t.shape[1], dtype=t.dtype, device="cuda")
    buf[:, -1] = t
    row = buf[:, -1]
    assert row.shape == t.shape and row.stride(0) == length * t.shape[1]
    return row


@pytest.mark.parametrize("where", ["x", "block"])
def test_residual_norm_in_place(where):
    g = gen(1)
    x, block = (randn(g, 1, 768).to(BF16) for _ in range(2))
    want = ops.residual_norm_forward(x, block, kind="rms")
    place = last_token(x if where == "x" else block)
    got = ops.residual_norm_forward(place if where == "x" else x, place if where == "block" else block, kind="rms", h=place)
    assert got[0] is place and all(same_bits(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("stride", [0, 8, 13, 1 << 45])
@pytest.mark.parametrize("out", [BF16, FP32])
def test_linear_cross_entropy_with_a_vocabulary_of_one(stride, out):
    _, hidden, table, _ = inputs(2, 200, 1, 72, BF16)
    labels = torch.zeros(200, dtype=torch.int64, device="cuda")
    place = torch.ones(72, dtype=out, device="cuda")
    for accumulate in (False, True):
        check(hidden, table.as_strided((1, 72), (stride, 1)), labels, dtable=place.as_strided((1, 72), (stride, 1)),
              accumulate=accumulate)


def test_linear_cross_entropy_of_one_row_in_place():
    _, hidden, table, labels = inputs(3, 1, 500, 72, BF16)
    want = ops.linear_cross_entropy(hidden, table, labels)
    row = last_token(hidden)
    got = ops.linear_cross_entropy(row, table, labels, dhidden=row)
    assert got[2] is row and all(same_bits(a, b) for a, b in zip(got, want))

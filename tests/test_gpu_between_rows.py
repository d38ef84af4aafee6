"""Matrices that lie between each other's rows, in one buffer, are apart: the same bits as in
buffers of their own."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_linear_loss import inputs
from test_gpu_operators import BF16, FP16, gen, randn, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def side_by_side(tensors):
    """The same values as columns of one buffer, neighbours without a gap."""
    buf = torch.cat(tensors, 1)
    at, out = 0, []
    for t in tensors:
        out.append(buf[:, at:at + t.shape[1]])
        at += t.shape[1]
    return out


def in_turns(tensors):
    """The same values as rows of one buffer, a row of each in turn."""
    buf = torch.stack(tensors, 1)
    return [buf[:, i] for i in range(len(tensors))]


@pytest.mark.parametrize("place", [side_by_side, in_turns])
@pytest.mark.parametrize("rows,cols,dtype", [(50, 768, BF16), (9, 77, FP16)])
def test_residual_norm(place, rows, cols, dtype):
    g = gen(1)
    x, block, h, y, dy, dx, dblock = (randn(g, rows, cols).to(dtype) for _ in range(7))
    want = ops.residual_norm_forward(x, block)
    grads = ops.residual_norm_backward(dy, None, want[0], block, want[2])
    x, block, h, y, dy, dx, dblock = place([x, block, h, y, dy, dx, dblock])
    got = ops.residual_norm_forward(x, block, h=h, y=y)
    assert got[0] is h and all(same_bits(a, b) for a, b in zip(got, want))
    back = ops.residual_norm_backward(dy, None, h, block, got[2], dx=dx, dblock=dblock)
    assert back[0] is dx and all(a is None and b is None or same_bits(a, b) for a, b in zip(back, grads))


@pytest.mark.parametrize("place", [side_by_side, in_turns])
@pytest.mark.parametrize("rows", [60, 200])
def test_linear_cross_entropy(place, rows):
    _, hidden, table, labels = inputs(2, rows, rows, 96, BF16)
    want = ops.linear_cross_entropy(hidden, table, labels)
    hidden, table, dhidden, dtable = place([hidden, table, torch.zeros_like(hidden), torch.zeros_like(table)])
    got = ops.linear_cross_entropy(hidden, table, labels, dhidden=dhidden, dtable=dtable)
    assert got[3] is dtable and all(same_bits(a, b) for a, b in zip(got, want))


def test_rows_of_several_strides_in_one_buffer():
    """x takes every second row of a buffer, h every fourth of the others."""
    g = gen(3)
    buf = randn(g, 64, 256).to(BF16)
    x, h = buf[:32:2], buf[1::4]
    block = randn(g, 16, 256).to(BF16)
    want = ops.residual_norm_forward(x.clone(), block)
    got = ops.residual_norm_forward(x, block, h=h)
    assert got[0] is h and all(same_bits(a, b) for a, b in zip(got, want))

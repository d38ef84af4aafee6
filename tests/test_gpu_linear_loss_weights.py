"""P's rounding to 16 bits does not move all of a gradient one way.

A mean gives every row the weight 1 / rows, and P at a label is close to minus that for each
of them: rounded as it is, 1 / 255 in bf16 is off by 2^-8 of itself in every row, and the
whole gradient of the table is too long by that much.  P counts in multiples of the largest
weight, so that there it is close to -1.

How far the gradient is off along the correctly rounded one: the results' own roundings
cancel there but for those that P's error tips over, which are as many up as down: with u
for each of n elements at the worst 6 u / sqrt(3 n), and n is 4000 or more; P at a label
loses at most q (5e-5 on average), which is what is left of -1 + q where it is rounded to -1.
All of it is less than u / 8.  (Along the gradient before its rounding the bound would not
hold: rows / 255 have the elements h (1 + 1 / 255) 2^-8 for h of eight bits, which are all
between half a step and a whole one above h, so that rounding moves them all up, by 1.1e-3
on average.)"""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_linear_loss import check, inputs, reference
from test_gpu_operators import BF16, FP16, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def along(got, want):
    want = want.to(got.dtype).double()
    return ((got.double() * want).sum() / want.square().sum() - 1.0).abs().item()


@pytest.mark.parametrize("dtype,rows", [(BF16, 85), (BF16, 255), (FP16, 2047)])
def test_a_mean_over_the_rows(dtype, rows):
    _, hidden, table, labels = inputs(rows, rows, 20000, 64, dtype, sharp=0.1)
    weight = torch.full((rows,), 1.0 / rows, device="cuda")
    scale = 65536.0 if dtype == FP16 else 1.0             # keeps fp16's gradients among its normal numbers
    want, _ = reference(hidden, table, labels, weight, scale)
    got = ops.linear_cross_entropy(hidden, table, labels, weight, grad_scale=scale)
    assert along(got[2], want[2]) <= U[dtype] / 8
    assert along(got[3], want[3]) <= U[dtype] / 8
    check(hidden, table, labels, weight, grad_scale=scale)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("size", [1e-41, 2.0 ** -130, 1e-30, 3e30, 3.3e38])
def test_weights_of_any_size(dtype, size):
    """The smallest and largest weights that fp32 has; grad_scale brings the gradients back to order 1."""
    _, hidden, table, labels = inputs(7, 150, 700, 64, dtype)
    weight = torch.full((150,), size, device="cuda")
    weight[::3] *= 0.4
    scale = min(1.0 / size, 3e38)
    want, _ = reference(hidden, table, labels, weight, scale)
    got = ops.linear_cross_entropy(hidden, table, labels, weight, grad_scale=scale)
    for a, b in zip(got[2:], want[2:]):
        assert torch.isfinite(a).all()
        # weights below 2^-126 (in fp16 below 2^-111) are held in fewer bits: multiples of 2^-126 2^-24 of P
        assert ((a.double() - b).norm() <= (2.0 ** -6 if size > 1e-40 else 2.0 ** -4) * b.norm())

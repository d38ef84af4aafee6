"""Waits of the head's products that run out at any point of a launch: every result is NaN or,
where none ran out, what it should be; nothing is left on its way, so that the next call is
right bit for bit.  Few steps of K let the copying warp finish before the others give up,
many let the two blocks of a pair stop at different stages."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_linear_loss import inputs
from test_gpu_operators import BF16, FP32, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("rows", [40, 128, 200, 1000])
@pytest.mark.parametrize("cols", [40, 200, 1500])
@pytest.mark.parametrize("out", [BF16, FP32])
def test_after_a_wait_that_ran_out(rows, cols, out):
    _, hidden, table, labels = inputs(rows + cols, rows, 30000, cols, BF16)
    dtable = lambda: torch.empty(30000, cols, dtype=out, device="cuda")  # noqa: E731
    want = ops.linear_cross_entropy(hidden, table, labels, dtable=dtable())
    for polls in (0, 1, 2, 5):
        for unit in (-1, 0, 3):
            B.so_debug_set_operator_polls(polls, unit)
            try:
                got = ops.linear_cross_entropy(hidden, table, labels, dtable=dtable())
            finally:
                B.so_debug_set_operator_polls(1 << 20)
            lost = [bool(torch.isnan(t).all()) for t in got]
            assert all(lost) or all(same_bits(a, b) for a, b in zip(got, want)), (polls, unit)
            assert polls or all(lost)
            got = ops.linear_cross_entropy(hidden, table, labels, dtable=dtable())
            assert all(same_bits(a, b) for a, b in zip(got, want)), (polls, unit)

"""Cross entropy from the hidden states with more tiles of both gradients than there are
blocks, so that a block ends tiles of dH and then tiles of dW, in each of the ways that dW
is written: dH has to be what it is alone, bit for bit, whatever dW does in between."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_linear_loss import check, inputs
from test_gpu_operators import BF16, FP16, FP32, randn, same_bits, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("rows,vocab,cols", [(300, 128256, 77), (100, 128256, 77), (3, 50257, 200), (128, 50257, 256), (700, 50257, 256)])
@pytest.mark.parametrize("dtype,out,accumulate", [(BF16, BF16, False), (BF16, BF16, True), (FP16, FP16, True), (FP16, BF16, True)])
def test_hidden_gradient_beside_the_tables(rows, vocab, cols, dtype, out, accumulate):
    g, hidden, table, labels = inputs(rows + cols, rows, vocab, cols, dtype)
    alone = ops.linear_cross_entropy(hidden, table, labels, dtable=False)
    kept = randn(g, vocab, cols).to(out) if accumulate else torch.zeros(vocab, cols, dtype=out, device="cuda")
    first = None
    for again in range(6):
        dtable = strided(kept, 1)                         # rows off 16-byte boundaries
        got = ops.linear_cross_entropy(hidden, table, labels, dtable=dtable, accumulate=accumulate)
        assert all(same_bits(a, b) for a, b in zip(got[:3], alone)), again
        first = dtable.clone() if first is None else first
        assert same_bits(dtable, first), again
    check(hidden, table, labels, dtable=kept.clone(), accumulate=accumulate)


@pytest.mark.parametrize("rows", [60, 9000])
@pytest.mark.parametrize("out", [BF16, FP32])
def test_accumulates_over_several_pieces(rows, out):
    """P of 9000 rows comes in two pieces of the vocabulary or more."""
    g, hidden, table, labels = inputs(31, rows, 20000, 136, BF16)
    check(hidden, table, labels, dtable=randn(g, 20000, 136).to(out), accumulate=True)
    check(hidden, table, labels, dtable=strided(randn(g, 20000, 136).to(out), 3, 1), accumulate=True)

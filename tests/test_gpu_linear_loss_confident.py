"""Cross entropy from the hidden states where a label has nearly all the probability: the
loss and P at the label are then 1 - q, six decimals below the numbers around them.

The logits are exact here: a row of hidden states is 1 in two columns of its own, the
table holds z's whole part in one and its rest, in eighths, in the other.  So errors
are those of what comes behind the logits.  With x = z - top exact and |x| <= 32, the
exponent x log2(e) takes two roundings of 2^-24 of at most 47 (3.9e-6 of the term), the
exponential 2^-22, and sums, quotient, logarithm and weight less than 2^-20 together:
everything is good to 2^-17 of itself (P at the label: of 1 - q).  An fp32 dtable adds
P's own bits: 24 (bf16), or 22 and multiples of 2^-39 of twice the weight (fp16)."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_operators import BF16, FP16, U, close, gen

pytestmark = pytest.mark.gpu
KINDS = [(top, left) for top in (25.0, 60.0, -30.0, 200.0, 131072.0) for left in (1e-2, 1e-4, 1e-6)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def inputs(rows, vocab, dtype):
    """A row for each of KINDS, the others masked: (hidden, table, labels, weight, logits in 64 bits)."""
    g = gen(rows + vocab)
    n = len(KINDS)
    kinds = [(min(top, 32768.0) if dtype == FP16 else top, left) for top, left in KINDS]
    hidden, table = torch.zeros(rows, 2 * n, device="cuda"), torch.zeros(vocab, 2 * n, device="cuda")
    labels = torch.full((rows,), -100, dtype=torch.int64, device="cuda")
    at = torch.randperm(rows, generator=g, device="cuda")[:n].sort()[0]
    labels[at] = torch.randperm(vocab, generator=g, device="cuda")[:n]
    z = torch.empty(n, vocab, dtype=torch.float64, device="cuda")
    for k, (top, left) in enumerate(kinds):
        below = math.log((vocab - 1) / left) + 2.0 * torch.rand(vocab, generator=g, device="cuda") - 1.0
        below = (8.0 * below).round() / 8.0
        below[labels[at[k]]] = 0.0
        hidden[at[k], 2 * k:2 * k + 2] = 1.0
        table[:, 2 * k], table[:, 2 * k + 1] = top, -below
        z[k] = top - below.double()
    assert torch.equal(table.to(dtype).float(), table)
    return hidden.to(dtype), table.to(dtype), labels, torch.full((rows,), 0.5, device="cuda"), at, z


# logits that are kept between the statistics and P, and ones that are not
@pytest.mark.parametrize("rows,vocab", [(20, 5000), (300, 3001), (20, 70001), (400, 50257)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_confident_labels(rows, vocab, dtype):
    hidden, table, labels, weight, at, z = inputs(rows, vocab, dtype)
    n = len(KINDS)
    dtable = torch.empty(vocab, 2 * n, device="cuda")
    _, row_loss, dhidden, _ = ops.linear_cross_entropy(hidden, table, labels, weight, dtable=dtable)
    label = labels[at][:, None]
    e = (z - z.gather(1, label)).exp().scatter_(1, label, 0.0)
    others = e.sum(1)
    left = others / (1.0 + others)                       # 1 - q of the label
    close(row_loss[at], torch.log1p(others), 2.0 ** -17 * others, "row_loss")
    p = 0.5 * e / (1.0 + others)[:, None]
    p.scatter_(1, label, -0.5 * left[:, None])
    got = dtable[:, ::2].t().contiguous()                # (each column has one row)
    assert torch.equal(dtable[:, ::2], dtable[:, 1::2])
    grain = 2.0 ** -40 if dtype == FP16 else 0.0
    close(got.gather(1, label), p.gather(1, label), 2.0 ** -17 * 0.5 * left[:, None] + grain, "P at the label")
    close(got, p, 2.0 ** -17 * p.abs() + grain, "P")
    # a row's P sums to nothing
    assert (got.double().sum(1).abs() <= 2.0 ** -17 * left + vocab * grain).all()
    # dH: P's terms are rounded to 16 bits but for the label's
    w, size = table.double(), p.abs()
    size = size.scatter(1, label, 0.0) * U[dtype] + 2.0 ** -17 * size + grain
    slack = size @ w.abs() + (vocab / 16 + 72) * 2.0 ** -22 * (p.abs() @ w.abs())
    close(dhidden[at], p @ w, slack, "dhidden")

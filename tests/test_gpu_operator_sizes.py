"""Sizes of the operators between the last block and the updated weights at which something
changes: more than 2^31 elements, both sides of the limits of what is kept or held in
registers, the widest rows, the most groups."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from paper_2509_21271_b200.tensor_adamw import TensorAdamW
from test_gpu_linear_loss import check, inputs
from test_gpu_operators import BF16, FP16, FP32, gen, randn, same_bits, strided
from test_gpu_residual_norm import Case
from test_gpu_tensor_adamw import HP

pytestmark = pytest.mark.gpu
BEYOND = (1 << 31) // 4096 + 40                           # rows of 4096: more than 2^31 elements


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()


def scratch(rows, vocab, cols, gradients):
    return B.so_linear_cross_entropy_scratch(rows, vocab, cols, B.SO_DTYPE_BF16, B.SO_DTYPE_BF16, gradients, 0)


@pytest.mark.parametrize("rows,cols,kept", [(1025, 768, True), (1300, 768, False), (250, 264, True), (300, 264, False)])
@pytest.mark.parametrize("out", [BF16, FP32])
def test_logits_that_are_kept_and_ones_that_are_not(rows, cols, kept, out):
    vocab = 50257
    logits = -(-rows // 256) * 256 * (-(-vocab // 256) * 256) * 4
    assert (scratch(rows, vocab, cols, 1) - scratch(rows, vocab, cols, 0) > logits) == kept
    _, hidden, table, labels = inputs(rows, rows, vocab, cols, BF16)
    check(hidden, table, labels, out=out)


@pytest.mark.parametrize("rows,vocab,cols", [(3, 10, 65536), (200, 300, 65536), (5, 2000, 30001)])
def test_widest_heads(rows, vocab, cols):
    _, hidden, table, labels = inputs(rows + vocab, rows, vocab, cols, FP16)
    check(hidden, table, labels, out=FP32)


@pytest.mark.parametrize("rows,pad", [(5, 0), (200, 0), (5, 1)])
def test_a_table_of_more_than_2_31_elements(rows, pad):
    """The table repeats 1024 rows: the softmax is one over these with their numbers as factors, and
    the gradients of the table are looked at in its beginning, middle and end."""
    cols = 4096
    g = gen(rows)
    hidden = (randn(g, rows, cols) * 0.25).to(BF16)
    few = (randn(g, 1024, cols) * 0.02).to(BF16)
    vocab = BEYOND
    table = torch.empty(vocab, cols + pad, dtype=BF16, device="cuda")[:, :cols]
    for at in range(0, vocab, 1024):
        table[at:at + 1024] = few[:min(1024, vocab - at)]
    labels = torch.randint(vocab - 100, vocab, (rows,), generator=g, device="cuda")
    labels[0] = 3
    loss, row_loss, dhidden, dtable = ops.linear_cross_entropy(hidden, table, labels)
    z = hidden.double() @ few.double().t()
    times = torch.full((1024,), float(vocab // 1024), dtype=torch.float64, device="cuda")
    times[:vocab % 1024] += 1
    lse = torch.logsumexp(z + times.log(), 1)
    own = z.gather(1, (labels % 1024)[:, None])[:, 0]
    # logits are good to (4096 / 16 + 8) 2^-22 of |h| |w|, which is below 20 here
    assert ((row_loss.double() - (lse - own)).abs() <= 264 * 2.0 ** -22 * 40).all()
    q = (z - lse[:, None]).exp()
    want = -few.double()[labels % 1024] + (q * times) @ few.double()
    size = few.double()[labels % 1024].abs() + (q * times) @ few.double().abs()
    assert ((dhidden.double() - want).abs() <= (2.0 ** -8 + 264 * 2.0 ** -21 * 20) * size).all()
    for lo, hi in ((0, 100), (vocab // 2, vocab // 2 + 50), (vocab - 100, vocab)):
        ids = torch.arange(lo, hi, device="cuda")
        p = q[:, ids % 1024].clone()
        p[labels[:, None] == ids] -= 1.0
        want, size = p.t() @ hidden.double(), p.abs().t() @ hidden.double().abs()
        assert ((dtable[lo:hi].double() - want).abs() <= (2.0 ** -7 + 264 * 2.0 ** -21 * 20) * size).all()


@pytest.mark.parametrize("pad", [0, 1])
def test_residual_norm_of_more_than_2_31_elements(pad):
    """The last rows are what they are by themselves, bit for bit."""
    g = gen(1)
    room = lambda: torch.empty(BEYOND, 4096 + pad, dtype=BF16, device="cuda")[:, :4096]  # noqa: E731
    x, block, h, y, dx, dblock = (room() for _ in range(6))
    for t in (x, block):
        t[:-60] = 1.0
        t[-60:] = randn(g, 60, 4096)
    w = randn(g, 4096)
    _, _, stats = ops.residual_norm_forward(x, block, None, None, None, w, h=h, y=y)
    none = dict(dweight=False, dbias=False)
    ops.residual_norm_backward(y, x, h, block, stats, None, None, None, w, dx=dx, dblock=dblock, **none)
    part = [strided(t[-60:], pad) for t in (x, block)]
    want = ops.residual_norm_forward(*part, None, None, None, w)
    assert all(same_bits(a, b) for a, b in zip((h[-60:], y[-60:], stats[:, -60:]), want))
    back = ops.residual_norm_backward(strided(want[1], pad), part[0], strided(want[0], pad), part[1], want[2], None, None, None, w, **none)
    assert same_bits(dx[-60:], back[0]) and same_bits(dblock[-60:], back[1])


@pytest.mark.parametrize("rows,cols,dtype", [(200, 8192, BF16), (150, 8208, BF16), (40, 12288, BF16), (33, 16384, FP16), (50, 7032, FP32),
                                             (50, 7044, FP32), (40, 6144, BF16), (40, 6152, BF16), (2, 300_001, BF16)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_residual_norm_around_the_widest_rows_in_registers(rows, cols, dtype, kind):
    Case(rows + cols, rows, cols, dtype, FP32, kind, groups=2 if rows % 2 == 0 else 1, biases=kind == "layer").check()


def test_as_many_gates_as_there_may_be():
    Case(2, 65535, 16, BF16, FP32, groups=65535).check()
    Case(3, 2 * 65535, 8, FP32, FP32, groups=65535).check()


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_on_a_tensor_of_more_than_2_31_elements(bits):
    """Its last elements are what they are in a tensor of their own, bit for bit."""
    n, tail = (1 << 31) + 5000, 3000
    first = (n - tail) // B.SO_TENSOR_BLOCK * B.SO_TENSOR_BLOCK
    g = gen(4)
    param, grad = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    param[first:], grad[first:] = randn(g, n - first), randn(g, n - first)
    own = TensorAdamW([param[first:].clone()], [grad[first:].clone()], state_bits=bits)
    opt = TensorAdamW([param], [grad], state_bits=bits)
    hp = HP(max_grad_norm=0.5)
    for _ in range(2):
        opt.step(hp)
        own.step(hp)
    assert abs(opt.stats[0].item() - own.stats[0].item()) <= 2.0 ** -22 * own.stats[0].item()
    assert same_bits(opt.stats[1:], own.stats[1:])
    assert same_bits(param[first:], own.params[0]) and (param[:first] == 0).all()
    at = first // B.SO_TENSOR_BLOCK * B.SO_TENSOR_BLOCK
    assert same_bits(opt.m[at:], own.m) and same_bits(opt.v[at:], own.v)

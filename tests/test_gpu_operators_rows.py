"""Losses on logits whose rows are far from even: elements that lie up to 88 nats
above what the kernels see of the row first, with weights as small as those of a
large batch.  References, tolerances and their derivation: ``test_gpu_operators``."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from test_gpu_operators import BF16, FP16, FP32, check_distill, check_policy, close, gen, path, randn, same_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


# 2^60 is 41.6 nats, 2^100 69.3, 2^128 88.7
HEIGHTS = (20.0, 30.0, 41.5, 43.0, 60.0, 70.0, 77.0, 80.0, 82.0, 85.0, 86.0, 88.5)


def uneven_rows(rows, vocab, dtype, temperature, kind, first):
    """Logits whose first `first` elements (or, at "shares", the first of every eighth) lie
    a height below the others; at "spikes" all are level but for a few."""
    h = torch.tensor(HEIGHTS, device="cuda")[torch.arange(rows, device="cuda") % len(HEIGHTS)] * temperature
    at = torch.arange(vocab, device="cuda")
    noise = 0.05 * temperature * randn(gen(rows + vocab), rows, vocab)
    if kind == "spikes":
        up = torch.zeros(vocab, dtype=torch.bool, device="cuda")
        up[torch.tensor([10_000, 20_000, 20_001, vocab - 9_000], device="cuda")] = True
        z = torch.where(up, h[:, None].expand(rows, vocab), noise)
    elif kind == "prefix":
        z = torch.where(at < first, -h[:, None], 0.0) + noise
    else:
        z = torch.where(at % (vocab // 8 + 1) < first, -h[:, None], 0.0) + noise
    return z.to(dtype)


# (rows, vocabulary): one block a row, two, eight
@pytest.mark.parametrize("rows,vocab", [(180, 50_257), (160, 128_256), (13, 128_256)])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("temperature", [1.0, 0.1])
@pytest.mark.parametrize("kind,first", [("spikes", 0), ("prefix", 2048), ("prefix", 4096), ("prefix", 8192), ("shares", 8192)])
def test_losses_of_rows_that_rise_above_what_is_seen_first(rows, vocab, dtype, temperature, kind, first):
    z = uneven_rows(rows, vocab, dtype, temperature, kind, first)
    ids = torch.tensor([3, 9_999, 10_000, 20_001, vocab - 1], device="cuda").expand(rows, 5).contiguous()
    teacher = randn(gen(8), rows, 5) * temperature
    # a mean over 8192 rows, as a loss scale carries it to fp16
    weight = torch.full((rows,), 1 / 8192, device="cuda")
    scale = 2.0 ** 20 if dtype == FP16 else 1.0
    check_distill(z, ids, teacher, weight, temperature, scale)
    check_distill(z, ids, teacher, weight, temperature, grad=False)
    tokens = ids[:, 2].clone()
    tokens[::2] = 3
    adv = randn(gen(9), rows)
    check_policy(z, tokens, adv, weight, temperature=temperature, grad_scale=scale)


@pytest.mark.parametrize("height", [40.0, 69.0, 77.0, 88.0])
@pytest.mark.parametrize("weight", [1e-6, 1e-12])
def test_small_weights_keep_the_gradients_digits(height, weight):
    """coef / S stays a normal number: fp32 gradients of rows whose sum is large against
    the first elements, with small coefficients."""
    z = torch.zeros(90, 50_257, device="cuda")
    z[:, :8192] = -height
    ids = torch.full((90, 1), 30_000, device="cuda")
    check_distill(z, ids, torch.zeros(90, 1, device="cuda"), torch.full((90,), weight, device="cuda"))
    check_policy(z, ids[:, 0].contiguous(), torch.ones(90, device="cuda"), torch.full((90,), weight, device="cuda"))


@pytest.mark.parametrize("dtype,vocab", [(FP16, 950_003), (BF16, 950_008), (FP32, 480_001)])
def test_vocabularies_that_no_cluster_holds(dtype, vocab):
    """More than 1.7 MB a row: the loop that reads a row twice, each type, in place and beside
    lists that are empty, repeat an id or are as long as they get."""
    g = gen(vocab)
    z = (randn(g, 5, vocab) * 2).to(dtype)
    ids = torch.randint(vocab, (5, 30), generator=g, device="cuda")
    ids[1, :] = -1                                # nothing there: counts as masked
    ids[2, 5:9] = ids[2, 4]
    teacher = randn(g, 5, 30)
    teacher[3, 7:] = -float("inf")
    weight = torch.tensor([1.0, 0.5, 0.25, 2.0, 0.0], device="cuda")
    scale = 512.0 if dtype == FP16 else 1.0
    _, row, grad = check_distill(z, ids, teacher, weight, 1.3, scale)
    assert row[1] == 0 and (grad[1] == 0).all()
    check_distill(z, ids[:, :1].repeat(1, 1024), randn(g, 5, 1024), weight, 1.0, scale)
    over = z.clone()
    check_distill(over, ids, teacher, weight, 1.3, scale, grad=over)
    assert same_bits(over, grad)
    tokens, adv = ids[:, 0].contiguous(), randn(g, 5)
    _, _, _, grad = check_policy(z, tokens, adv, weight, temperature=0.8, grad_scale=scale)
    over = z.clone()
    check_policy(over, tokens, adv, weight, temperature=0.8, grad_scale=scale, grad=over)
    assert same_bits(over, grad)


def test_lookup_of_the_widest_rows():
    """Rows of 2^31 - 1 elements: the last step of the loop over columns ends beyond 2^31."""
    cols = 2 ** 31 - 1
    table = torch.empty(1, cols, dtype=FP16, device="cuda")
    table.view(torch.int16).random_(0, 0x7C00)       # finite, every magnitude
    out = ops.embedding_forward(torch.zeros(1, dtype=torch.int64, device="cuda"), table)
    assert torch.equal(out.view(torch.int16), table.view(torch.int16))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("vocab", [517, 50_257])
@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_targets_masked_with_the_types_lowest_value(dtype, vocab, rows, temperature):
    """log q is then the lowest value over T: a number in nats, none in units of log2."""
    g = gen(vocab + rows)
    z = (randn(g, rows, vocab) * 2).to(dtype)
    ids = (5 + 7 * torch.arange(6, device="cuda")).expand(rows, 6).contiguous()
    z[:, 5] = torch.finfo(dtype).min
    z[1] = torch.finfo(dtype).min                 # a row of nothing else: uniform
    teacher = randn(g, rows, 6)
    weight = torch.full((rows,), 1 / rows, device="cuda")
    _, row, grad = check_distill(z, ids, teacher, weight, temperature)
    assert torch.isfinite(row).all() and torch.isfinite(grad).all() and (row[0] > 1e36).all()
    check_distill(z, ids, teacher, weight, temperature, grad=False)
    tokens, adv = ids[:, 0].contiguous(), torch.ones(rows, device="cuda")
    _, _, logp, _ = check_policy(z, tokens, adv, weight, temperature=temperature)
    assert torch.isfinite(logp).all()
    # sampled under the same logits: the ratio is 1 and nothing is infinite
    loss, row, again, grad = ops.policy_loss(z, tokens, adv, weight, old_logp=logp, ref_logp=logp, kl_coef=0.1,
                                             temperature=temperature)
    assert same_bits(again, logp) and (row == -1).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("vocab", [517, 50_257, 480_001])
@pytest.mark.parametrize("high", [0.2, float("inf")])
def test_no_advantage_is_no_loss_however_large_the_ratio(vocab, high):
    """exp(logp - old_logp) is infinite in fp32 beyond 88.7; times 0 it is still 0."""
    z = randn(gen(vocab), 4, vocab)
    tokens = torch.tensor([0, 5, 300, vocab - 1], device="cuda")
    old = torch.tensor([-200.0, -99.0, -1e4, -1e30], device="cuda")
    adv = torch.tensor([0.0, -0.0, 0.0, 0.0], device="cuda")
    loss, row, logp, grad = ops.policy_loss(z, tokens, adv, old_logp=old, clip_high=high)
    assert (row == 0).all() and (loss == 0).all() and (grad == 0).all()
    adv[1], z[2, 7] = -1.0, float("nan")          # a loss with a ratio like that, and NaN, stay what they are
    loss, row, logp, grad = ops.policy_loss(z, tokens, adv, old_logp=old, clip_high=high)
    assert row[0] == 0 and torch.isnan(row[2]) and torch.isnan(grad[2]).all()
    # the difference rounds to 2^-24 of some 90, the exponential to 2^-22
    ratio = (logp[1].double() - old[1].double()).exp()
    assert row[1] == float("inf") if ratio > torch.finfo(FP32).max else abs(row[1].double() - ratio) <= 1e-5 * ratio


@pytest.mark.parametrize("offset", [-7.5, 9.0, 300.0, 1e4, 1e6])
@pytest.mark.parametrize("rows,cols", [(70, 768), (33, 4096), (40, 515), (9, 5000), (5, 9000)])
def test_layer_norm_backward_of_rows_far_from_zero(rows, cols, offset):
    """x - mean first, as the formula has it: its rounding is relative to the difference, not
    to x.  fp32, whose outputs would show it; the mean and rstd are inputs, taken as given."""
    g = gen(rows + cols)
    x, dy, w = randn(g, rows, cols) + offset, randn(g, rows, cols) * 0.1, 1 + 0.2 * randn(g, cols)
    _, mean, rstd = ops.layer_norm_forward(x)
    dx, dw, db = ops.layer_norm_backward(dy, x, mean, rstd, w)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    gw, r = dy.double() * w.double(), rstd.double()[:, None]
    want = r * (gw - gw.mean(1, keepdim=True) - xh * (gw * xh).mean(1, keepdim=True))
    size = r * (gw.abs() + gw.abs().mean(1, keepdim=True) + xh.abs() * (gw * xh).abs().mean(1, keepdim=True))
    close(dx, want, path(cols) * size, "dx")
    close(dw, (dy.double() * xh).sum(0), path(rows) * (dy.double() * xh).abs().sum(0), "dweight")
    close(db, dy.double().sum(0), path(rows) * dy.double().abs().sum(0), "dbias")

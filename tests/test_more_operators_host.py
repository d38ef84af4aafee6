"""Argument checks of the C entry points for the loss from the hidden states, the norms on
both sides of a residual and AdamW over a list of tensors, and their sizes: all of it is
decided before anything is launched, so no GPU is needed.  Addresses are made up; only
refusals are called."""
from __future__ import annotations

import ctypes as C

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops
from paper_2509_21271_b200.tensor_adamw import TensorAdamW
from test_operators_host import A, BF16, FP16, FP32, INF, NAN, refused, variants


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()


LINEAR = dict(hidden=A, hidden_stride=64, table=2 * A, table_stride=64, labels=A, ids_dtype=B.SO_IDS_INT64, weight=A, rows=5,
              vocab=100, cols=64, dtype=BF16, grad_scale=1.0, dhidden=3 * A, dhidden_stride=64, dtable=4 * A, dtable_stride=64,
              grad_dtype=FP32, accumulate=0, row_loss=A, loss=A, scratch=5 * A, scratch_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(LINEAR, [
    ("hidden", None), ("hidden", A + 1), ("hidden_stride", 63), ("hidden_stride", -64), ("table", None), ("table", A + 1),
    ("table_stride", 63), ("table_stride", 0), ("labels", None), ("labels", A + 4), ("ids_dtype", 2), ("weight", A + 2),
    ("rows", -1), ("rows", 2 ** 22 + 1), ("vocab", 0), ("vocab", 2 ** 26 + 1), ("cols", 0), ("cols", 2 ** 16 + 1),
    ("dtype", FP32), ("dtype", 3), ("grad_scale", NAN), ("grad_scale", INF), ("grad_scale", 1e39), ("dhidden", A + 1),
    ("dhidden", 2 * A), ("dhidden_stride", 0), ("dhidden_stride", 63), ("dtable", 4 * A + 2), ("dtable", 2 * A),
    ("dtable", A), ("dtable", 3 * A), ("dtable_stride", 63), ("grad_dtype", 3), ("accumulate", 2), ("row_loss", None),
    ("row_loss", A + 2), ("loss", None), ("loss", A + 1), ("scratch", None), ("scratch", A + 16), ("scratch_bytes", 1000),
    ("table_stride", 2 ** 60)])))
def test_linear_cross_entropy_refuses(name, value, args):
    assert refused(B.so_linear_cross_entropy, *args)


def test_linear_cross_entropy_in_place_needs_one_stride():
    assert refused(B.so_linear_cross_entropy, *dict(LINEAR, dhidden=A, dhidden_stride=72).values())


def test_linear_cross_entropy_scratch():
    size = lambda *a: B.so_linear_cross_entropy_scratch(*a)  # noqa: E731
    alone, with_gradients = size(8192, 128256, 4096, BF16, BF16, 0, 0), size(8192, 128256, 4096, BF16, BF16, 1, 0)
    # far below the logits' 2.1 GB; the hidden states once more, and statistics, for the loss alone
    assert 8192 * 4096 * 2 < alone < 128 << 20 and alone < with_gradients < 512 << 20
    assert size(8192, 128256, 4096, BF16, BF16, 0, 1) > alone
    assert size(0, 1, 1, FP16, FP32, 1, 1) > 0
    short = dict(LINEAR, scratch_bytes=size(5, 100, 64, BF16, FP32, 1, 0) - 1)
    assert refused(B.so_linear_cross_entropy, *short.values())
    for bad in ((-1, 10, 10, BF16, BF16, 1, 0), (1, 0, 10, BF16, BF16, 1, 0), (1, 10, 0, BF16, BF16, 1, 0), (1, 10, 10, FP32, BF16, 1, 0),
                (1, 10, 10, BF16, 5, 1, 0), (1, 10, 10, BF16, BF16, 2, 0), (1, 10, 10, BF16, BF16, 1, 7)):
        assert refused(B.so_linear_cross_entropy_scratch, *bad)


FORWARD = dict(x=A, x_stride=96, block=2 * A, block_stride=96, gate=A, groups=2, post_weight=A, post_bias=A, weight=A, bias=A, h=3 * A,
               h_stride=96, y=4 * A, y_stride=96, stats=A, rows=6, cols=96, dtype=FP16, param_dtype=FP32, kind=B.SO_NORM_LAYER,
               post=1, scale=1.0, eps=1e-5, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(FORWARD, [
    ("x", None), ("x", A + 1), ("x_stride", 95), ("block", None), ("block", A + 1), ("block_stride", -1), ("gate", A + 2), ("groups", 0),
    ("groups", 4), ("groups", 65536), ("post_weight", A + 2), ("post_bias", A + 1), ("weight", A + 2), ("bias", A + 1), ("h", None),
    ("h", 4 * A), ("h", 3 * A + 1), ("h_stride", 0), ("y", None), ("y", A), ("y", 2 * A), ("y_stride", 95), ("stats", A + 2), ("rows", -1),
    ("cols", 0), ("cols", 2 ** 31), ("dtype", 4), ("param_dtype", BF16), ("kind", 2), ("post", 2), ("post", 0), ("scale", NAN),
    ("scale", 1e39), ("eps", -1.0), ("eps", NAN), ("eps", INF)])))
def test_residual_norm_forward_refuses(name, value, args):
    assert refused(B.so_residual_norm_forward, *args)


@pytest.mark.parametrize("h,stride", [(A, 104), (2 * A, 104)])
def test_residual_norm_in_place_needs_one_stride(h, stride):
    assert refused(B.so_residual_norm_forward, *dict(FORWARD, h=h, h_stride=stride).values())


BACKWARD = dict(dy=A, dy_stride=96, dh=A, dh_stride=96, h=A, h_stride=96, block=A, block_stride=96, stats=A, gate=A, groups=2, post_weight=A,
                post_bias=A, weight=A, dx=2 * A, dx_stride=96, dblock=3 * A, dblock_stride=96, dgate=A, dpost_weight=A, dpost_bias=A,
                dweight=A, dbias=A, rows=6, cols=96, dtype=BF16, param_dtype=BF16, grad_dtype=FP32, kind=B.SO_NORM_RMS, post=1,
                accumulate=0, scale=1.0, scratch=A, scratch_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(BACKWARD, [
    ("dy", None), ("dy", A + 1), ("dy_stride", 95), ("dh", A + 1), ("dh_stride", 10), ("h", None), ("h", 2 * A), ("block", None),
    ("block", 3 * A), ("stats", None), ("stats", A + 1), ("gate", A + 1), ("groups", 5), ("groups", 0), ("post_weight", A + 1),
    ("weight", A + 1), ("dx", None), ("dx", 3 * A), ("dx", A), ("dx_stride", 0), ("dblock", None), ("dblock", A), ("dblock_stride", 90),
    ("dgate", A + 2), ("dpost_weight", A + 1), ("dpost_bias", A + 2), ("dweight", A + 1), ("dbias", A + 2), ("rows", -2), ("cols", 0),
    ("dtype", -1), ("param_dtype", FP16), ("grad_dtype", 3), ("kind", -1), ("post", 0), ("accumulate", 2), ("scale", INF),
    ("scratch", None), ("scratch", A + 8), ("scratch_bytes", 64)])))
def test_residual_norm_backward_refuses(name, value, args):
    assert refused(B.so_residual_norm_backward, *args)


def test_residual_norm_scratch():
    assert 0 < B.so_residual_norm_backward_scratch(1, 768, 1) < B.so_residual_norm_backward_scratch(4096, 768, 1)
    for bad in ((-1, 768, 1), (4, 0, 1), (4, 768, 0), (4, 768, 3)):
        assert refused(B.so_residual_norm_backward_scratch, *bad)


HP = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, max_grad_norm=1.0)


def adamw(hyper=None, tensor=None, **kw):
    entry = dict(dict(param=A, grad=A, copy=A, numel=1000), **(tensor or {}))
    args = dict(tensors=(B.so_tensor * 2)(B.so_tensor(**entry), B.so_tensor(None, None, None, 0)), n=2, grad_dtype=BF16, copy_dtype=FP16,
                state_bits=8, m=A, v=A, m_scale=A, v_scale=A, hp=C.byref(B.so_hparams(**dict(HP, **(hyper or {})))), grad_scale=1.0, clip=1,
                stochastic=1, seed=5, record=A, scratch=A, scratch_bytes=1 << 30, stream=None)
    args.update(kw)
    return list(args.values())


@pytest.mark.parametrize("kw", [
    dict(tensors=None), dict(n=-1), dict(grad_dtype=3), dict(copy_dtype=FP32), dict(copy_dtype=-2), dict(state_bits=16), dict(m=None),
    dict(v=None), dict(m=A + 16), dict(m_scale=None), dict(v_scale=None), dict(hp=None), dict(grad_scale=NAN), dict(grad_scale=1e39),
    dict(clip=2), dict(stochastic=-1), dict(state_bits=32), dict(record=None), dict(record=A + 8), dict(scratch=None),
    dict(scratch=A + 8), dict(scratch_bytes=8), dict(tensor=dict(param=None)), dict(tensor=dict(param=A + 2)), dict(tensor=dict(grad=None)),
    dict(tensor=dict(grad=A + 1)), dict(tensor=dict(copy=None)), dict(tensor=dict(copy=A + 1)), dict(tensor=dict(numel=-1)),
    dict(tensor=dict(numel=2 ** 62)), dict(hyper=dict(lr=-1.0)), dict(hyper=dict(lr=NAN)), dict(hyper=dict(lr=1e39)), dict(hyper=dict(beta1=1.0)),
    dict(hyper=dict(beta1=-0.1)), dict(hyper=dict(beta2=NAN)), dict(hyper=dict(eps=0.0)), dict(hyper=dict(eps=1e-60)), dict(hyper=dict(eps=INF)),
    dict(hyper=dict(weight_decay=-1.0)), dict(hyper=dict(weight_decay=1e60)), dict(hyper=dict(max_grad_norm=NAN))],
    ids=lambda kw: "-".join(f"{k}={v}" for k, v in kw.items()))
def test_tensor_adamw_refuses(kw):
    assert refused(B.so_tensor_adamw_step, *adamw(**kw))


def test_tensor_adamw_layout_and_moments():
    sizes = [1, 256, 257, 0, 100_000]
    tensors = (B.so_tensor * 5)(*[B.so_tensor(None, None, None, n) for n in sizes])
    info = B.so_tensor_adamw_layout(tensors, 5, 8)
    assert info.blocks == 1 + 1 + 2 + 0 + 391 and info.bytes_moment == info.blocks * 256 and info.bytes_scale == info.blocks
    wide = B.so_tensor_adamw_layout(tensors, 5, 32)
    assert wide.bytes_moment == 4 * info.bytes_moment and wide.bytes_scale == 0 and wide.bytes_record == info.bytes_record
    for bad in ((None, 5, 8), (tensors, -1, 8), (tensors, 5, 4)):
        assert refused(B.so_tensor_adamw_layout, *bad)
    good = dict(m=A, v=A, m_scale=A, v_scale=A, blocks=3, m_out=A, v_out=A, stream=None)
    for name, value, args in variants(good, [("m", None), ("m", A + 4), ("v", None), ("m_scale", None), ("v_scale", None), ("blocks", -1),
                                             ("blocks", 2 ** 40), ("m_out", None), ("v_out", A + 8)]):
        assert refused(B.so_tensor_adamw_moments, *args), (name, value)


def test_tensors_that_are_not_on_a_gpu_or_require_grad_are_refused():
    x, ids = torch.zeros(2, 8, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64)
    r = torch.zeros(2, 8, dtype=torch.bfloat16, requires_grad=True)
    for call in (lambda: ops.linear_cross_entropy(x, x, ids), lambda: ops.residual_norm_forward(x, x),
                 lambda: ops.residual_norm_backward(x, x, x, x, x), lambda: TensorAdamW([x], [x])):
        with pytest.raises(B.SuperOffloadError, match="CUDA device"):
            call()
    for call in (lambda: ops.linear_cross_entropy(r, x, ids), lambda: ops.linear_cross_entropy(x, r, ids),
                 lambda: ops.linear_cross_entropy(x, x, ids, r[:, 0]), lambda: ops.residual_norm_forward(r, x),
                 lambda: ops.residual_norm_forward(x, r), lambda: ops.residual_norm_forward(x, x, r[0]),
                 lambda: ops.residual_norm_forward(x, x, None, r[0]), lambda: ops.residual_norm_backward(r, x, x, x, x),
                 lambda: ops.residual_norm_backward(x, r, x, x, x), lambda: ops.residual_norm_backward(x, x, x, x, x, r[0])):
        with pytest.raises(B.SuperOffloadError, match="requires grad") as err:
            call()
        assert err.value.status == B.SO_ERR_INVALID_ARG

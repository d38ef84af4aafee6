"""Argument checks of the operators' C entry points, and their scratch sizes: all of
it is decided before anything is launched, so no GPU is needed.  Addresses are
made up; an accepted call would try to launch, so only refusals are called."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops

BF16, FP32, FP16 = B.SO_DTYPE_BF16, B.SO_DTYPE_FP32, B.SO_DTYPE_FP16
A = 0x10000000                                    # an aligned address
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()


def refused(fn, *args):
    with pytest.raises(B.SuperOffloadError) as err:
        fn(*args)
    return err.value.status == B.SO_ERR_INVALID_ARG


def variants(good: dict, bad):
    """The good arguments with one of them replaced, for every (name, value)."""
    for name, value in bad:
        args = dict(good)
        assert name in args
        args[name] = value
        yield name, value, list(args.values())


NORM_FORWARD = dict(x=A, x_stride=768, weight=A, bias=A, y=2 * A, y_stride=768, mean=A, rstd=A, rows=4, cols=768,
                    dtype=BF16, param_dtype=BF16, eps=1e-5, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(NORM_FORWARD, [
    ("x", None), ("x", A + 1), ("x_stride", 767), ("weight", A + 1), ("bias", A + 1), ("y", None), ("y", 2 * A + 1),
    ("y_stride", 767), ("y_stride", 0), ("mean", None), ("rstd", None), ("mean", A + 2), ("rows", -1), ("cols", 0),
    ("cols", -5), ("cols", 2 ** 31), ("dtype", 3), ("dtype", -1), ("param_dtype", FP16), ("eps", -1e-5), ("eps", NAN),
    ("eps", INF), ("x_stride", 2 ** 62)])))
def test_layer_norm_forward_refuses(name, value, args):
    assert refused(B.so_layer_norm_forward, *args)


def test_layer_norm_forward_in_place_needs_one_stride():
    args = dict(NORM_FORWARD, y=A, y_stride=800)
    assert refused(B.so_layer_norm_forward, *args.values())


NORM_BACKWARD = dict(dy=A, dy_stride=768, x=A, x_stride=768, weight=A, mean=A, rstd=A, dx=2 * A, dx_stride=768,
                     dweight=A, dbias=A, rows=4, cols=768, dtype=FP16, param_dtype=FP32, grad_dtype=FP32,
                     accumulate=0, scratch=A, scratch_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(NORM_BACKWARD, [
    ("dy", None), ("dy", A + 1), ("dy_stride", 10), ("x", None), ("x_stride", 767), ("weight", A + 2), ("mean", None),
    ("rstd", None), ("dx", None), ("dx_stride", 0), ("dweight", A + 2), ("dbias", A + 1), ("rows", -2), ("cols", 0),
    ("dtype", 7), ("param_dtype", BF16), ("grad_dtype", 9), ("accumulate", 2), ("scratch", None), ("scratch", A + 8),
    ("scratch_bytes", 100)])))
def test_layer_norm_backward_refuses(name, value, args):
    assert refused(B.so_layer_norm_backward, *args)


EMBEDDING_FORWARD = dict(ids=A, ids_dtype=B.SO_IDS_INT64, n=5, table=A, table_stride=64, vocab=100, cols=64, dtype=FP32,
                         scale=1.0, out=2 * A, out_stride=64, bad_id=None, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(EMBEDDING_FORWARD, [
    ("ids", None), ("ids", A + 4), ("ids_dtype", 2), ("n", -1), ("n", 2 ** 30 + 1), ("table", None), ("table", A + 2),
    ("table_stride", 63), ("vocab", 0), ("vocab", 2 ** 30 + 1), ("cols", 0), ("dtype", 5), ("scale", NAN),
    ("scale", INF), ("out", None), ("out_stride", 0), ("bad_id", A + 1)])))
def test_embedding_forward_refuses(name, value, args):
    assert refused(B.so_embedding_forward, *args)


EMBEDDING_BACKWARD = dict(ids=A, ids_dtype=B.SO_IDS_INT32, n=5, dout=A, dout_stride=64, vocab=100, cols=64, dtype=BF16,
                          scale=1.0, padding_id=-1, dtable=2 * A, dtable_stride=64, grad_dtype=FP32, accumulate=0,
                          scratch=A, scratch_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(EMBEDDING_BACKWARD, [
    ("ids", None), ("ids", A + 2), ("ids_dtype", -1), ("n", -1), ("dout", None), ("dout", A + 1), ("dout_stride", 5),
    ("vocab", 0), ("cols", 0), ("dtype", 4), ("scale", NAN), ("dtable", None), ("dtable", 2 * A + 2),
    ("dtable_stride", 0), ("grad_dtype", 3), ("accumulate", -1), ("scratch", None), ("scratch", A + 4),
    ("scratch_bytes", 64)])))
def test_embedding_backward_refuses(name, value, args):
    assert refused(B.so_embedding_backward, *args)


DISTILL = dict(logits=A, logits_stride=1000, teacher_ids=A, ids_dtype=B.SO_IDS_INT32, ids_stride=8, teacher_logits=A,
               teacher_stride=8, teacher_dtype=FP32, top_k=8, weight=None, rows=3, vocab=1000, dtype=BF16,
               temperature=1.0, grad_scale=1.0, grad=2 * A, grad_stride=1000, row_loss=A, loss=A, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(DISTILL, [
    ("logits", None), ("logits", A + 1), ("logits_stride", 999), ("teacher_ids", None), ("teacher_ids", A + 2),
    ("ids_dtype", 4), ("ids_stride", 7), ("teacher_logits", None), ("teacher_logits", A + 2), ("teacher_stride", 7),
    ("teacher_dtype", 3), ("top_k", 0), ("top_k", B.SO_DISTILL_MAX_TOP_K + 1), ("weight", A + 1), ("rows", -1),
    ("vocab", 0), ("vocab", 2 ** 31), ("dtype", 3), ("temperature", 0.0), ("temperature", -1.0), ("temperature", NAN),
    ("temperature", INF), ("temperature", 1e-60), ("temperature", 1e60), ("grad_scale", NAN), ("grad_scale", INF),
    ("grad_scale", 1e60), ("grad", 2 * A + 1), ("grad_stride", 0), ("grad_stride", 999), ("row_loss", None),
    ("row_loss", A + 2), ("loss", None), ("loss", A + 1)])))
def test_distill_loss_refuses(name, value, args):
    assert refused(B.so_distill_loss, *args)


POLICY = dict(logits=A, logits_stride=1000, tokens=A, ids_dtype=B.SO_IDS_INT64, advantage=A, old_logp=A, ref_logp=A,
              weight=A, rows=3, vocab=1000, dtype=FP32, temperature=0.7, clip_low=0.2, clip_high=0.2, kl_coef=0.1,
              grad_scale=1.0, grad=2 * A, grad_stride=1000, logp=A, row_loss=A, loss=A, stream=None)


@pytest.mark.parametrize("name,value,args", list(variants(POLICY, [
    ("logits", None), ("logits", A + 2), ("tokens", None), ("tokens", A + 4), ("advantage", None), ("advantage", A + 1),
    ("old_logp", A + 1), ("ref_logp", None), ("ref_logp", A + 2), ("weight", A + 2), ("rows", -3), ("temperature", 0.0),
    ("clip_low", -0.1), ("clip_low", 1.1), ("clip_low", NAN), ("clip_high", -0.1), ("clip_high", NAN),
    ("kl_coef", -1.0), ("kl_coef", NAN), ("kl_coef", INF), ("grad", 2 * A + 2), ("grad_stride", 10), ("logp", A + 2),
    ("row_loss", None), ("loss", None)])))
def test_policy_loss_refuses(name, value, args):
    assert refused(B.so_policy_loss, *args)


@pytest.mark.parametrize("which", [DISTILL, POLICY])
def test_losses_in_place_need_one_stride(which):
    fn = B.so_distill_loss if which is DISTILL else B.so_policy_loss
    assert refused(fn, *dict(which, grad=A, grad_stride=1008).values())


def test_scratch_sizes_grow_with_the_problem_and_refuse_nonsense():
    assert B.so_layer_norm_backward_scratch(0, 768) >= 2 * 768 * 4
    small, large = B.so_layer_norm_backward_scratch(10, 768), B.so_layer_norm_backward_scratch(100_000, 768)
    assert 0 < small < large == B.so_layer_norm_backward_scratch(10_000_000, 768)
    assert B.so_embedding_backward_scratch(0, 50257, 768) < B.so_embedding_backward_scratch(8192, 50257, 768)
    for fn, args in ((B.so_layer_norm_backward_scratch, (-1, 768)), (B.so_layer_norm_backward_scratch, (4, 0)),
                     (B.so_embedding_backward_scratch, (-1, 10, 10)), (B.so_embedding_backward_scratch, (4, 0, 10)),
                     (B.so_embedding_backward_scratch, (4, 2 ** 31, 10))):
        assert refused(fn, *args)


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x, ids = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: ops.layer_norm_forward(x), lambda: ops.layer_norm_backward(x, x, x[:, 0], x[:, 0]),
                 lambda: ops.embedding_forward(ids, x), lambda: ops.embedding_backward(ids, x, x),
                 lambda: ops.distill_loss(x, ids[:, None], x[:, :1]), lambda: ops.policy_loss(x, ids, x[:, 0])):
        with pytest.raises(B.SuperOffloadError, match="CUDA device"):
            call()


@pytest.mark.parametrize("polls,unit", [(-1, -1), (2 ** 20 + 1, -1), (2 ** 40, 0), (5, -2)])
def test_operator_polls_refuse(polls, unit):
    assert refused(B.so_debug_set_operator_polls, polls, unit)


def test_tensors_that_require_grad_are_refused():
    """Their result would be cut off from the graph without a word."""
    x, ids = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64)
    r = torch.zeros(2, 8, requires_grad=True)
    calls = [lambda: ops.layer_norm_forward(r), lambda: ops.layer_norm_forward(x, r[0]),
             lambda: ops.layer_norm_forward(x, x[0], r[0]), lambda: ops.layer_norm_backward(r, x, x[:, 0], x[:, 0]),
             lambda: ops.layer_norm_backward(x, x, x[:, 0], x[:, 0], r[0]), lambda: ops.embedding_forward(ids, r),
             lambda: ops.embedding_backward(ids, r, x), lambda: ops.distill_loss(r, ids[:, None], x[:, :1]),
             lambda: ops.distill_loss(x, ids[:, None], r[:, :1]), lambda: ops.policy_loss(r, ids, x[:, 0]),
             lambda: ops.policy_loss(x, ids, r[:, 0]), lambda: ops.policy_loss(x, ids, x[:, 0], r[:, 0])]
    for call in calls:
        with pytest.raises(B.SuperOffloadError, match="requires grad") as err:
            call()
        assert err.value.status == B.SO_ERR_INVALID_ARG
        with torch.no_grad(), pytest.raises(B.SuperOffloadError, match="CUDA device"):
            call()                                # the next check: these are not on a GPU


@pytest.mark.parametrize("which", [DISTILL, POLICY])
@pytest.mark.parametrize("vocab", [1, 1000, 200_000])
def test_losses_refuse_more_rows_than_a_grid_has_blocks(which, vocab):
    fn = B.so_distill_loss if which is DISTILL else B.so_policy_loss
    assert refused(fn, *dict(which, rows=2 ** 31, vocab=vocab, logits_stride=vocab, grad_stride=vocab).values())


@pytest.mark.parametrize("fn,good,name,value", [
    (B.so_layer_norm_forward, NORM_FORWARD, "eps", 1e39), (B.so_embedding_forward, EMBEDDING_FORWARD, "scale", 1e39),
    (B.so_embedding_forward, EMBEDDING_FORWARD, "scale", -1e300), (B.so_embedding_backward, EMBEDDING_BACKWARD, "scale", 4e38),
    (B.so_policy_loss, POLICY, "kl_coef", 1e60), (B.so_distill_loss, DISTILL, "temperature", 4e-39),
    (B.so_policy_loss, POLICY, "temperature", 3e-39)])
def test_scalars_that_fp32_does_not_hold_are_refused(fn, good, name, value):
    """They are finite as given; in fp32 they, or log2(e) / T, are not."""
    assert refused(fn, *dict(good, **{name: value}).values())

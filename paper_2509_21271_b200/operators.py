"""Operators of a training step around its matrix products, on torch tensors.

Token embedding, layer norm, the norms on both sides of a residual, and the losses
on the logits, each with its gradient; every one is a call of the C ABI (``include/superoffload.h`` has the
formulas and the rules on strides, types and masked rows).  Torch allocates the
results that the caller does not bring and names the stream, nothing else.

Gradients of parameters may be written straight into views of a
``BucketedAdamW`` gradient arena: any of bf16, fp16, fp32, whatever the
activations' type.

Every function runs on the current stream, or on ``stream`` (a
``torch.cuda.Stream``; the tensors it is given are then recorded on it, ordering
it behind their producers is the caller's).  Tensors live on the current device.
Nothing here waits for the device.

Autograd does not record these calls: the backward passes are calls of their own.
With gradients enabled an input that requires grad is refused rather than cut off
from its graph; call them under ``torch.no_grad()`` or from a
``torch.autograd.Function``.  Tensors that are written over (``out=x``,
``grad=logits``, gradients added to) count as modified in place, so that a graph
which saved one of them notices.
"""
from __future__ import annotations

from functools import lru_cache

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.SO_DTYPE_BF16, torch.float32: B.SO_DTYPE_FP32, torch.float16: B.SO_DTYPE_FP16}
_IDS = {torch.int32: B.SO_IDS_INT32, torch.int64: B.SO_IDS_INT64}


# The plain forms of these go through Python layers that cost as much as a launch.
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)
_increment_version = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version


def _refuse(where: str, what: str):
    raise B.SuperOffloadError(B.SO_ERR_INVALID_ARG, f"{where}: {what}")


def _recorded(where):
    """Some input requires grad: refused where autograd would be expected to record the call."""
    if torch.is_grad_enabled():
        _refuse(where, "autograd does not record this call, and a tensor given to it requires grad: "
                       "use torch.no_grad() or a torch.autograd.Function")


def _device(where, name, t) -> int:
    """The current device's index, on which `t` has to be."""
    dev = t.get_device()
    if dev < 0:
        _refuse(where, f"{name} is not on a CUDA device")
    if dev != _current_device():
        _refuse(where, f"{name} is not on the current device")
    return dev


def _dtype(where, name, t) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        _refuse(where, f"{name} has dtype {t.dtype}: bfloat16, float16 and float32 are supported")
    return code


def _ids_dtype(where, name, t) -> int:
    code = _IDS.get(t.dtype)
    if code is None:
        _refuse(where, f"{name} has dtype {t.dtype}: int32 and int64 are supported")
    return code


def _rows(where, name, t, dev):
    """(rows, cols, row stride) of a tensor seen as a matrix of its last dimension."""
    if t.get_device() != dev:
        _refuse(where, f"{name} is not on the current CUDA device")
    shape = t.shape
    dim = len(shape)
    if dim == 2:
        rows, cols = shape
        stride, step = t.stride()
    elif dim == 1:
        rows, cols, stride, step = 1, shape[0], shape[0], t.stride(0)
    elif dim > 2 and t.is_contiguous():
        cols = shape[-1]
        rows, stride, step = (t.numel() // cols if cols else 0), cols, 1
    else:
        _refuse(where, f"{name} must be a matrix, or contiguous with more dimensions")
    if step != 1 and cols > 1:
        _refuse(where, f"the elements of {name}'s rows must be contiguous")
    return rows, cols, stride


def _vector(where, name, t, n, dev, dtype=None):
    """The address of a contiguous vector of n elements (None passes)."""
    if t is None:
        return None
    if t.get_device() != dev:
        _refuse(where, f"{name} is not on the current CUDA device")
    if t.numel() != n or not t.is_contiguous():
        _refuse(where, f"{name} must be contiguous with {n} elements")
    if dtype is not None and t.dtype != dtype:
        _refuse(where, f"{name} must be {dtype}")
    return t.data_ptr()


def _same(where, name, t, like_name, like):
    if t.shape != like.shape or t.dtype != like.dtype:
        _refuse(where, f"{name} must have the shape and dtype of {like_name}")


def _scratch(where, scratch, dev):
    if scratch.get_device() != dev or not scratch.is_contiguous():
        _refuse(where, "scratch must be contiguous on the current CUDA device")
    return scratch.numel() * scratch.element_size()


_norm_scratch = lru_cache(maxsize=512)(B.so_layer_norm_backward_scratch)      # sizes alone decide
_embedding_scratch = lru_cache(maxsize=512)(B.so_embedding_backward_scratch)
_residual_scratch = lru_cache(maxsize=512)(B.so_residual_norm_backward_scratch)
_linear_scratch = lru_cache(maxsize=512)(B.so_linear_cross_entropy_scratch)
_KINDS = {"layer": B.SO_NORM_LAYER, "rms": B.SO_NORM_RMS}


def _done(status: int, where: str, written) -> None:
    """Raises, or notes that the tensors in `written` were."""
    if status != B.SO_OK:
        raise B.SuperOffloadError(status, "so_" + where)
    _increment_version(written)


def _on_stream(stream, fn, *args, **kw):
    """The call on another stream than the current one; its tensors are recorded there."""
    with torch.cuda.stream(stream):
        out = fn(*args, **kw)
    for t in (*args, *kw.values()):
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
    return out


# ---- layer norm ----------------------------------------------------------------

def layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, *, out=None, mean=None, rstd=None,
                       save_stats: bool = True, stream=None):
    """y = (x - mean) * rstd * weight + bias over the last dimension; returns
    (y, mean, rstd).  `weight` and `bias` are of x's dtype or fp32.  `out` may be
    `x`.  With ``save_stats=False`` mean and rstd are not written (None)."""
    if stream is not None:
        return _on_stream(stream, layer_norm_forward, x, weight, bias, eps, out=out, mean=mean, rstd=rstd,
                          save_stats=save_stats)
    where = "layer_norm_forward"
    if x.requires_grad or weight is not None and weight.requires_grad or bias is not None and bias.requires_grad:
        _recorded(where)
    dev = _device(where, "x", x)
    dt = _dtype(where, "x", x)
    rows, cols, stride = _rows(where, "x", x, dev)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _same(where, "out", out, "x", x)
    _, _, out_stride = _rows(where, "out", out, dev)
    pt = dt
    first = weight if weight is not None else bias
    if first is not None:
        pt = _dtype(where, "weight", first)
    wp = _vector(where, "weight", weight, cols, dev)
    bp = _vector(where, "bias", bias, cols, dev, None if first is None else first.dtype)
    if save_stats:
        if mean is None:
            mean = torch.empty(rows, dtype=torch.float32, device=x.device)
        if rstd is None:
            rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    elif mean is not None or rstd is not None:
        _refuse(where, "mean and rstd are not written with save_stats=False")
    _done(B.lib().so_layer_norm_forward(x.data_ptr(), stride, wp, bp, out.data_ptr(), out_stride,
                            _vector(where, "mean", mean, rows, dev, torch.float32),
                            _vector(where, "rstd", rstd, rows, dev, torch.float32),
                            rows, cols, dt, pt, eps, _raw_stream(dev)), where, (out, mean, rstd) if save_stats else (out,))
    return out, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, *, dx=None, dweight=None, dbias=None,
                        accumulate: bool = False, scratch=None, stream=None):
    """Gradients of the forward pass; returns (dx, dweight, dbias).  `dweight` and
    `dbias` are written (with `accumulate`: added to) where given, in their own
    dtype, allocated in weight's (or x's) dtype where None, and not computed where
    False.  `dx` may be `dy`.  `scratch`: so_layer_norm_backward_scratch bytes."""
    if stream is not None:
        return _on_stream(stream, layer_norm_backward, dy, x, mean, rstd, weight, dx=dx, dweight=dweight,
                          dbias=dbias, accumulate=accumulate, scratch=scratch)
    where = "layer_norm_backward"
    if dy.requires_grad or x.requires_grad or weight is not None and weight.requires_grad:
        _recorded(where)
    dev = _device(where, "x", x)
    dt = _dtype(where, "x", x)
    _same(where, "dy", dy, "x", x)
    rows, cols, stride = _rows(where, "x", x, dev)
    _, _, dy_stride = _rows(where, "dy", dy, dev)
    if dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _same(where, "dx", dx, "x", x)
    _, _, dx_stride = _rows(where, "dx", dx, dev)
    pt = dt if weight is None else _dtype(where, "weight", weight)
    if accumulate and (dweight is None or dbias is None):
        _refuse(where, "accumulate needs dweight and dbias (or False)")
    kind = x.dtype if weight is None else weight.dtype
    if dweight is None:
        dweight = torch.empty(cols, dtype=kind, device=x.device)
    if dbias is None:
        dbias = torch.empty(cols, dtype=kind, device=x.device)
    dweight = None if dweight is False else dweight
    dbias = None if dbias is False else dbias
    gt, need, ws = dt, 0, None
    if dweight is not None or dbias is not None:
        some = dweight if dweight is not None else dbias
        gt = _dtype(where, "dweight", some)
        if dweight is not None and dbias is not None and dbias.dtype != dweight.dtype:
            _refuse(where, "dweight and dbias must have one dtype")
        if scratch is None:
            scratch = torch.empty(_norm_scratch(rows, cols), dtype=torch.uint8, device=x.device)
        need, ws = _scratch(where, scratch, dev), scratch.data_ptr()
    _done(B.lib().so_layer_norm_backward(dy.data_ptr(), dy_stride, x.data_ptr(), stride,
                             _vector(where, "weight", weight, cols, dev),
                             _vector(where, "mean", mean, rows, dev, torch.float32),
                             _vector(where, "rstd", rstd, rows, dev, torch.float32),
                             dx.data_ptr(), dx_stride, _vector(where, "dweight", dweight, cols, dev),
                             _vector(where, "dbias", dbias, cols, dev), rows, cols, dt, pt, gt, int(accumulate),
                             ws, need, _raw_stream(dev)), where,
          [t for t in (dx, dweight, dbias) if t is not None])
    return dx, dweight, dbias


# ---- the norms on both sides of a residual ------------------------------------------

def _param(where, name, t, n, dev, dtype):
    """_vector's address of a parameter; its checks one by one only where something is wrong."""
    if t is None:
        return None
    if t.dtype is dtype and t.numel() == n and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    return _vector(where, name, t, n, dev, dtype)


def _gate(where, gate, cols):
    """How many gates there are."""
    if gate is None or gate.dim() == 1 and gate.shape[0] == cols:
        return 1
    if gate.dim() != 2 or gate.shape[1] != cols:
        _refuse(where, "gate must be a row, or a matrix of one row per group of rows")
    return gate.shape[0]


def _like(where, name, t, like_name, like, dev, rows, cols):
    """Row stride of a matrix with the shape and dtype of `like`."""
    if t.shape != like.shape or t.dtype != like.dtype:
        _same(where, name, t, like_name, like)
    if t.get_device() == dev and t.is_contiguous():
        return cols
    return _rows(where, name, t, dev)[2]


def residual_norm_forward(x, block, gate=None, post_weight=None, post_bias=None, weight=None, bias=None, *,
                          kind: str = "layer", post: bool = True, scale: float = 1.0, eps: float = 1e-5, h=None,
                          y=None, stats=None, save_stats: bool = True, stream=None):
    """What lies between two blocks: with u the norm of `block` (times `post_weight`,
    plus `post_bias`), or `block` itself where `post` is False,
    h = scale * x + gate * u and y = norm(h) * weight + bias; returns (h, y, stats).

    `kind` is "layer" or "rms".  `gate` is a row, or [groups, cols] with a row for each
    of `groups` equal runs of rows; the parameters have one dtype, x's or fp32.  `h` may
    be `x` or `block`.  `stats` (fp32 [4, rows]) is for the backward pass; None with
    ``save_stats=False``."""
    if stream is not None:
        return _on_stream(stream, residual_norm_forward, x, block, gate, post_weight, post_bias, weight, bias,
                          kind=kind, post=post, scale=scale, eps=eps, h=h, y=y, stats=stats, save_stats=save_stats)
    where = "residual_norm_forward"
    if x.requires_grad or block.requires_grad or gate is not None and gate.requires_grad \
            or post_weight is not None and post_weight.requires_grad or post_bias is not None and post_bias.requires_grad \
            or weight is not None and weight.requires_grad or bias is not None and bias.requires_grad:
        _recorded(where)
    dev = _device(where, "x", x)
    dt = _dtype(where, "x", x)
    rows, cols, stride = _rows(where, "x", x, dev)
    block_stride = _like(where, "block", block, "x", x, dev, rows, cols)
    if kind not in _KINDS:
        _refuse(where, "kind is 'layer' or 'rms'")
    if h is None:
        h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    h_stride = _like(where, "h", h, "x", x, dev, rows, cols)
    y_stride = _like(where, "y", y, "x", x, dev, rows, cols)
    groups = _gate(where, gate, cols)
    first = gate if gate is not None else post_weight if post_weight is not None else post_bias if post_bias is not None \
        else weight if weight is not None else bias
    kept = x.dtype if first is None else first.dtype
    pt = dt if first is None else _dtype(where, "a parameter", first)
    if not save_stats:
        if stats is not None:
            _refuse(where, "stats are not written with save_stats=False")
    elif stats is None:
        stats = torch.empty(4, rows, dtype=torch.float32, device=x.device)
    _done(B.lib().so_residual_norm_forward(
        x.data_ptr(), stride, block.data_ptr(), block_stride, _param(where, "gate", gate, groups * cols, dev, kept), groups,
        _param(where, "post_weight", post_weight, cols, dev, kept), _param(where, "post_bias", post_bias, cols, dev, kept),
        _param(where, "weight", weight, cols, dev, kept), _param(where, "bias", bias, cols, dev, kept), h.data_ptr(),
        h_stride, y.data_ptr(), y_stride, _param(where, "stats", stats, 4 * rows, dev, torch.float32), rows, cols, dt, pt,
        _KINDS[kind], post, scale, eps, _raw_stream(dev)), where, (h, y) if stats is None else (h, y, stats))
    return h, y, stats


def residual_norm_backward(dy, dh, h, block, stats, gate=None, post_weight=None, post_bias=None, weight=None, *,
                           kind: str = "layer", post: bool = True, scale: float = 1.0, dx=None, dblock=None,
                           dgate=None, dpost_weight=None, dpost_bias=None, dweight=None, dbias=None,
                           accumulate: bool = False, scratch=None, stream=None):
    """Gradients of the forward pass from `dy` and `dh` (the residual stream's own; None:
    nothing); returns (dx, dblock, dgate, dpost_weight, dpost_bias, dweight, dbias).

    The parameters' gradients are written (with `accumulate`: added to) where given, of
    one dtype, and not computed where False.  Where None they are allocated in the
    parameters' dtype: dgate, dpost_weight and dpost_bias if that parameter is given,
    dweight always, dbias with the layer norm.  `scratch`:
    so_residual_norm_backward_scratch bytes."""
    if stream is not None:
        return _on_stream(stream, residual_norm_backward, dy, dh, h, block, stats, gate, post_weight, post_bias, weight,
                          kind=kind, post=post, scale=scale, dx=dx, dblock=dblock, dgate=dgate,
                          dpost_weight=dpost_weight, dpost_bias=dpost_bias, dweight=dweight, dbias=dbias,
                          accumulate=accumulate, scratch=scratch)
    where = "residual_norm_backward"
    if dy.requires_grad or h.requires_grad or block.requires_grad or dh is not None and dh.requires_grad \
            or gate is not None and gate.requires_grad or post_weight is not None and post_weight.requires_grad \
            or post_bias is not None and post_bias.requires_grad or weight is not None and weight.requires_grad:
        _recorded(where)
    dev = _device(where, "h", h)
    dt = _dtype(where, "h", h)
    rows, cols, h_stride = _rows(where, "h", h, dev)
    dy_stride = _like(where, "dy", dy, "h", h, dev, rows, cols)
    block_stride = _like(where, "block", block, "h", h, dev, rows, cols)
    dh_stride = 0 if dh is None else _like(where, "dh", dh, "h", h, dev, rows, cols)
    if kind not in _KINDS:
        _refuse(where, "kind is 'layer' or 'rms'")
    if dx is None:
        dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    if dblock is None:
        dblock = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    dx_stride = _like(where, "dx", dx, "h", h, dev, rows, cols)
    dblock_stride = _like(where, "dblock", dblock, "h", h, dev, rows, cols)
    groups = _gate(where, gate, cols)
    first = gate if gate is not None else post_weight if post_weight is not None else post_bias if post_bias is not None \
        else weight
    kept = h.dtype if first is None else first.dtype
    pt = dt if first is None else _dtype(where, "a parameter", first)
    if accumulate and (dgate is None and gate is not None or dpost_weight is None and post_weight is not None
                       or dpost_bias is None and post_bias is not None or dweight is None
                       or dbias is None and kind == "layer"):
        _refuse(where, "accumulate needs the gradients to add to (or False)")
    if gate is None and dgate is not None and dgate is not False:
        _refuse(where, "there is no gate to have a gradient")
    new = lambda shape: torch.empty(shape, dtype=kept, device=h.device)  # noqa: E731
    dgate = None if dgate is False else new(gate.shape) if dgate is None and gate is not None else dgate
    dpost_weight = None if dpost_weight is False else new(cols) if dpost_weight is None and post_weight is not None \
        else dpost_weight
    dpost_bias = None if dpost_bias is False else new(cols) if dpost_bias is None and post_bias is not None else dpost_bias
    dweight = None if dweight is False else new(cols) if dweight is None else dweight
    dbias = None if dbias is False else new(cols) if dbias is None and kind == "layer" else dbias
    out = (dx, dblock, dgate, dpost_weight, dpost_bias, dweight, dbias)
    some = dweight if dweight is not None else dgate if dgate is not None else dpost_weight if dpost_weight is not None \
        else dpost_bias if dpost_bias is not None else dbias
    gt, need, ws, kind_of = dt, 0, None, None
    if some is not None:
        kind_of = some.dtype
        gt = _dtype(where, "a parameter's gradient", some)
        if scratch is None:
            scratch = torch.empty(_residual_scratch(rows, cols, groups), dtype=torch.uint8, device=h.device)
        need, ws = _scratch(where, scratch, dev), scratch.data_ptr()
    _done(B.lib().so_residual_norm_backward(
        dy.data_ptr(), dy_stride, None if dh is None else dh.data_ptr(), dh_stride, h.data_ptr(), h_stride,
        block.data_ptr(), block_stride, _param(where, "stats", stats, 4 * rows, dev, torch.float32),
        _param(where, "gate", gate, groups * cols, dev, kept), groups, _param(where, "post_weight", post_weight, cols, dev, kept),
        _param(where, "post_bias", post_bias, cols, dev, kept), _param(where, "weight", weight, cols, dev, kept),
        dx.data_ptr(), dx_stride, dblock.data_ptr(), dblock_stride, _param(where, "dgate", dgate, groups * cols, dev, kind_of),
        _param(where, "dpost_weight", dpost_weight, cols, dev, kind_of), _param(where, "dpost_bias", dpost_bias, cols, dev, kind_of),
        _param(where, "dweight", dweight, cols, dev, kind_of), _param(where, "dbias", dbias, cols, dev, kind_of), rows, cols, dt,
        pt, gt, _KINDS[kind], post, accumulate, scale, ws, need, _raw_stream(dev)), where,
        [t for t in out if t is not None])
    return out


# ---- embedding -------------------------------------------------------------------

def embedding_forward(ids, table, scale: float = 1.0, *, out=None, bad_id=None, stream=None):
    """out[..., :] = scale * table[ids[...], :].  An id outside the table gives a
    row of zeros and sets `bad_id` (int32, one element), if given, to 1."""
    if stream is not None:
        return _on_stream(stream, embedding_forward, ids, table, scale, out=out, bad_id=bad_id)
    where = "embedding_forward"
    if table.requires_grad:
        _recorded(where)
    dev = _device(where, "table", table)
    it = _ids_dtype(where, "ids", ids)
    dt = _dtype(where, "table", table)
    if table.dim() != 2:
        _refuse(where, "table must be a matrix")
    vocab, cols, stride = _rows(where, "table", table, dev)
    n = ids.numel()
    ip = _vector(where, "ids", ids, n, dev)
    if out is None:
        out = torch.empty((*ids.shape, cols), dtype=table.dtype, device=table.device)
    elif out.shape != (*ids.shape, cols) or out.dtype != table.dtype:
        _refuse(where, "out must have the shape of ids with a row of the table each, and its dtype")
    _, _, out_stride = _rows(where, "out", out, dev)
    _done(B.lib().so_embedding_forward(ip, it, n, table.data_ptr(), stride, vocab, cols, dt, scale, out.data_ptr(),
                           out_stride, _vector(where, "bad_id", bad_id, 1, dev, torch.int32),
                           _raw_stream(dev)), where, (out,) if bad_id is None else (out, bad_id))
    return out


def embedding_backward(ids, dout, dtable, scale: float = 1.0, *, padding_id: int = -1,
                       accumulate: bool = False, scratch=None, stream=None):
    """dtable[v, :] = scale * sum of dout[t, :] over the tokens with id v, in
    `dtable`'s dtype; rows of ids that do not occur become zero, or with
    `accumulate` keep what they hold while the others are added to.  Tokens of
    `padding_id`, and ids outside the table, take no part.  `scratch`:
    so_embedding_backward_scratch bytes."""
    if stream is not None:
        return _on_stream(stream, embedding_backward, ids, dout, dtable, scale, padding_id=padding_id,
                          accumulate=accumulate, scratch=scratch)
    where = "embedding_backward"
    if dout.requires_grad or dtable.requires_grad:
        _recorded(where)
    dev = _device(where, "dtable", dtable)
    it = _ids_dtype(where, "ids", ids)
    dt = _dtype(where, "dout", dout)
    gt = _dtype(where, "dtable", dtable)
    if dtable.dim() != 2:
        _refuse(where, "dtable must be a matrix")
    vocab, cols, stride = _rows(where, "dtable", dtable, dev)
    n = ids.numel()
    ip = _vector(where, "ids", ids, n, dev)
    if dout.shape != (*ids.shape, cols):
        _refuse(where, "dout must have the shape of ids with a row of the table each")
    _, _, dout_stride = _rows(where, "dout", dout, dev)
    if scratch is None:
        scratch = torch.empty(_embedding_scratch(n, vocab, cols), dtype=torch.uint8, device=dtable.device)
    _done(B.lib().so_embedding_backward(ip, it, n, dout.data_ptr(), dout_stride, vocab, cols, dt, scale, padding_id,
                            dtable.data_ptr(), stride, gt, int(accumulate), scratch.data_ptr(),
                            _scratch(where, scratch, dev), _raw_stream(dev)), where, (dtable,))
    return dtable


# ---- losses on the logits ----------------------------------------------------------

def _loss_outputs(where, logits, rows, grad, loss, row_loss, dev):
    """(grad or None, its stride, loss, row_loss)."""
    if grad is None:
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    grad_stride = 0
    if grad is False:
        grad = None
    else:
        _same(where, "grad", grad, "logits", logits)
        _, _, grad_stride = _rows(where, "grad", grad, dev)
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=logits.device)
    if row_loss is None:
        row_loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    return grad, grad_stride, loss, row_loss


def distill_loss(logits, teacher_ids, teacher_logits, weight=None, *, temperature: float = 1.0,
                 grad_scale: float = 1.0, grad=None, loss=None, row_loss=None,
                 stream=None):
    """Distillation from a teacher's top logits; returns (loss, row_loss, grad).

    `logits` [rows, vocab], `teacher_ids` and `teacher_logits` [rows, top_k],
    `weight` fp32 [rows] (None: 1 each; 0 masks a row).  `grad` None allocates the
    gradient, False leaves it out, and a tensor, which may be `logits` itself,
    receives it, multiplied by `grad_scale`.  An entry of logit -inf, or an id
    outside the vocabulary, is empty."""
    if stream is not None:
        return _on_stream(stream, distill_loss, logits, teacher_ids, teacher_logits, weight,
                          temperature=temperature, grad_scale=grad_scale, grad=grad, loss=loss, row_loss=row_loss)
    where = "distill_loss"
    if logits.requires_grad or teacher_logits.requires_grad or weight is not None and weight.requires_grad:
        _recorded(where)
    dev = _device(where, "logits", logits)
    dt = _dtype(where, "logits", logits)
    rows, vocab, stride = _rows(where, "logits", logits, dev)
    it = _ids_dtype(where, "teacher_ids", teacher_ids)
    tt = _dtype(where, "teacher_logits", teacher_logits)
    ids_rows, top_k, ids_stride = _rows(where, "teacher_ids", teacher_ids, dev)
    t_rows, t_k, t_stride = _rows(where, "teacher_logits", teacher_logits, dev)
    if ids_rows != rows or t_rows != rows or t_k != top_k:
        _refuse(where, "teacher_ids and teacher_logits must have one row of top_k entries per row of logits")
    grad, grad_stride, loss, row_loss = _loss_outputs(where, logits, rows, grad, loss, row_loss, dev)
    _done(B.lib().so_distill_loss(logits.data_ptr(), stride, teacher_ids.data_ptr(), it, ids_stride,
                      teacher_logits.data_ptr(), t_stride, tt, top_k,
                      _vector(where, "weight", weight, rows, dev, torch.float32), rows, vocab, dt, temperature,
                      grad_scale, None if grad is None else grad.data_ptr(), grad_stride,
                      _vector(where, "row_loss", row_loss, rows, dev, torch.float32),
                      _vector(where, "loss", loss, 1, dev, torch.float32), _raw_stream(dev)), where,
          (loss, row_loss) if grad is None else (loss, row_loss, grad))
    return loss, row_loss, grad


def policy_loss(logits, tokens, advantage, weight=None, *, old_logp=None, ref_logp=None,
                temperature: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2,
                kl_coef: float = 0.0, grad_scale: float = 1.0, grad=None, loss=None, row_loss=None,
                logp=None, stream=None):
    """Clipped policy loss with a KL term, from the logits; returns (loss,
    row_loss, logp, grad).

    One row per sampled token: `tokens` [rows], `advantage`, `old_logp` (None:
    sampled from these logits), `ref_logp` (None: no KL term) and `weight` fp32
    [rows] (None: 1 each; 0 masks a row, as does a token outside the
    vocabulary).  `grad` and `grad_scale` as in :func:`distill_loss`."""
    if stream is not None:
        return _on_stream(stream, policy_loss, logits, tokens, advantage, weight, old_logp=old_logp,
                          ref_logp=ref_logp, temperature=temperature, clip_low=clip_low, clip_high=clip_high,
                          kl_coef=kl_coef, grad_scale=grad_scale, grad=grad, loss=loss, row_loss=row_loss, logp=logp)
    where = "policy_loss"
    if logits.requires_grad or any(t is not None and t.requires_grad for t in (advantage, weight, old_logp, ref_logp)):
        _recorded(where)
    dev = _device(where, "logits", logits)
    dt = _dtype(where, "logits", logits)
    rows, vocab, stride = _rows(where, "logits", logits, dev)
    it = _ids_dtype(where, "tokens", tokens)
    grad, grad_stride, loss, row_loss = _loss_outputs(where, logits, rows, grad, loss, row_loss, dev)
    if logp is None:
        logp = torch.empty(rows, dtype=torch.float32, device=logits.device)
    f32 = torch.float32
    _done(B.lib().so_policy_loss(logits.data_ptr(), stride, _vector(where, "tokens", tokens, rows, dev), it,
                     _vector(where, "advantage", advantage, rows, dev, f32),
                     _vector(where, "old_logp", old_logp, rows, dev, f32),
                     _vector(where, "ref_logp", ref_logp, rows, dev, f32),
                     _vector(where, "weight", weight, rows, dev, f32), rows, vocab, dt, temperature, clip_low,
                     clip_high, kl_coef, grad_scale, None if grad is None else grad.data_ptr(), grad_stride,
                     _vector(where, "logp", logp, rows, dev, f32), _vector(where, "row_loss", row_loss, rows, dev, f32),
                     _vector(where, "loss", loss, 1, dev, f32), _raw_stream(dev)), where,
          (loss, row_loss, logp) if grad is None else (loss, row_loss, logp, grad))
    return loss, row_loss, logp, grad


# ---- the loss from the hidden states -------------------------------------------------

def linear_cross_entropy(hidden, table, labels, weight=None, *, grad_scale: float = 1.0, dhidden=None, dtable=None,
                         accumulate: bool = False, loss=None, row_loss=None, scratch=None, stream=None):
    """Cross entropy of `labels` under the logits hidden @ table.T, which never leave
    the scratch (whole only where 256 MB hold them); returns (loss, row_loss, dhidden, dtable).

    `hidden` [rows, cols] and `table` [vocab, cols] are bfloat16 or float16, `labels`
    [rows], `weight` fp32 [rows] (None: 1 each; 0 masks a row, as does a label outside
    the vocabulary).  The gradients, multiplied by `grad_scale`, are allocated where
    None, left out where False, and written where a tensor is given: `dhidden` may be
    `hidden` itself, `dtable` has a dtype of its own and with `accumulate` is added to.
    `scratch`: so_linear_cross_entropy_scratch bytes on a 256-byte boundary."""
    if stream is not None:
        return _on_stream(stream, linear_cross_entropy, hidden, table, labels, weight, grad_scale=grad_scale,
                          dhidden=dhidden, dtable=dtable, accumulate=accumulate, loss=loss, row_loss=row_loss,
                          scratch=scratch)
    where = "linear_cross_entropy"
    if hidden.requires_grad or table.requires_grad or weight is not None and weight.requires_grad:
        _recorded(where)
    dev = _device(where, "hidden", hidden)
    dt = _dtype(where, "hidden", hidden)
    if dt == B.SO_DTYPE_FP32:
        _refuse(where, "hidden has dtype torch.float32: bfloat16 and float16 are supported")
    if table.dtype != hidden.dtype:
        _refuse(where, "table must have the dtype of hidden")
    if table.dim() != 2:
        _refuse(where, "table must be a matrix")
    rows, cols, stride = _rows(where, "hidden", hidden, dev)
    vocab, table_cols, table_stride = _rows(where, "table", table, dev)
    if table_cols != cols:
        _refuse(where, "table must have rows as long as hidden's")
    it = _ids_dtype(where, "labels", labels)
    lp = _vector(where, "labels", labels, rows, dev)
    if dhidden is None:
        dhidden = torch.empty(hidden.shape, dtype=hidden.dtype, device=hidden.device)
    elif dhidden is False:
        dhidden = None
    else:
        _same(where, "dhidden", dhidden, "hidden", hidden)
    if dtable is None:
        if accumulate:
            _refuse(where, "accumulate needs dtable (or False)")
        dtable = torch.empty(table.shape, dtype=table.dtype, device=table.device)
    elif dtable is False:
        dtable = None
    elif dtable.shape != table.shape:
        _refuse(where, "dtable must have the shape of table")
    dhidden_stride = dtable_stride = 0
    gt = dt
    if dhidden is not None:
        _, _, dhidden_stride = _rows(where, "dhidden", dhidden, dev)
    if dtable is not None:
        _, _, dtable_stride = _rows(where, "dtable", dtable, dev)
        gt = _dtype(where, "dtable", dtable)
    if loss is None:
        loss = torch.empty(1, dtype=torch.float32, device=hidden.device)
    if row_loss is None:
        row_loss = torch.empty(rows, dtype=torch.float32, device=hidden.device)
    tp = table.data_ptr()
    if scratch is None:
        packed = tp % 16 != 0 or vocab > 1 and table_stride % 8 != 0
        scratch = torch.empty(_linear_scratch(rows, vocab, cols, dt, gt, int(dhidden is not None or dtable is not None),
                                              int(packed)), dtype=torch.uint8, device=hidden.device)
    f32 = torch.float32
    _done(B.lib().so_linear_cross_entropy(
        hidden.data_ptr(), stride, tp, table_stride, lp, it, _vector(where, "weight", weight, rows, dev, f32), rows, vocab,
        cols, dt, grad_scale, None if dhidden is None else dhidden.data_ptr(), dhidden_stride,
        None if dtable is None else dtable.data_ptr(), dtable_stride, gt, int(accumulate),
        _vector(where, "row_loss", row_loss, rows, dev, f32), _vector(where, "loss", loss, 1, dev, f32), scratch.data_ptr(),
        _scratch(where, scratch, dev), _raw_stream(dev)), where,
        [t for t in (loss, row_loss, dhidden, dtable) if t is not None])
    return loss, row_loss, dhidden, dtable

"""AdamW over a list of tensors where they lie, moments in 32 or in 8 bits.

``TensorAdamW`` is the optimizer for parameters that do not live in a
``BucketedAdamW`` arena: one pass over fp32 tensors and their gradients, wherever
torch has them, clipped by the global norm and skipped where that is not finite.
With ``state_bits=8`` the moments take 2 bytes a parameter in place of 8
(``include/superoffload.h`` has the formulas and the code).  Torch allocates the
moments and names the stream, nothing else; every step runs in the library's
kernels, and nothing here waits for the device but ``step_count``.
"""
from __future__ import annotations

import ctypes as C
from bisect import bisect_left
from typing import Optional, Sequence

import torch

from . import binding as B
from .operators import _DTYPES, _current_device, _increment_version, _raw_stream, _refuse

_data_ptr = torch.Tensor.data_ptr


class TensorAdamW:
    """The moments and the progress of AdamW over `params`.

    `params` are contiguous fp32 tensors, `grads` contiguous and of one dtype (bf16,
    fp16 or fp32), `copies` (None: none) bf16 or fp16; each list has the same sizes, on
    the current device.  Parameters and copies are apart from each other and from the
    gradients, which may share memory with each other.  The optimizer keeps them; gradients are read where they are
    when :meth:`step` runs.  A tensor that has been given other storage
    (``p.data = other``) is taken up with it by the next step, and refused there where it no
    longer fits; a captured step goes on with the storage of its capture, which the caller
    keeps.  Parameters may require grad: a step counts as a modification in place.

    `m` and `v` are arenas of blocks of 256 elements, every tensor from a block of its
    own on (:meth:`block_of`): fp32, or codes with a byte of scale per block in
    `m_scale` and `v_scale`.  Zeros are a fresh start.  A checkpoint is these arenas,
    the parameters and :meth:`step_count`.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], *,
                 copies: Optional[Sequence[torch.Tensor]] = None, state_bits: int = 32):
        where = "TensorAdamW"
        if state_bits not in (8, 32):
            _refuse(where, "state_bits is 8 or 32")
        self.params = list(params)
        self.copies = None if copies is None else list(copies)
        self.state_bits = state_bits
        n = len(self.params)
        if n == 0:
            _refuse(where, "there is no tensor")
        self.device = self.params[0].device
        if self.device.type != "cuda":
            _refuse(where, "the parameters are not on a CUDA device")
        if self.device.index != _current_device():
            _refuse(where, "the parameters are not on the current device")
        self._list = (B.so_tensor * n)()
        self._numels = [p.numel() for p in self.params]
        for e, numel in zip(self._list, self._numels):
            e.numel = numel
        self._copy_dtype = B.SO_TENSOR_NO_COPY
        if self.copies is not None:
            dtypes = {c.dtype for c in self.copies}
            if len(self.copies) != n or len(dtypes) != 1 or not dtypes <= {torch.bfloat16, torch.float16}:
                _refuse(where, "there must be a copy for each parameter, all bfloat16 or all float16")
            self._copy_dtype = _DTYPES[self.copies[0].dtype]
        self.grads = None
        self._take_written(where)
        self.set_grads(grads)
        info = B.so_tensor_adamw_layout(self._list, n, state_bits)
        self.blocks = info.blocks
        kind = torch.float32 if state_bits == 32 else torch.uint8
        zeros = lambda size, dtype: torch.zeros(size, dtype=dtype, device=self.device)  # noqa: E731
        self.m, self.v = (zeros(self.blocks * B.SO_TENSOR_BLOCK, kind) for _ in range(2))
        self.m_scale, self.v_scale = (zeros(self.blocks, torch.uint8) if state_bits == 8 else None for _ in range(2))
        self._record = zeros(info.bytes_record, torch.uint8)
        self._scratch = zeros(info.bytes_scratch, torch.uint8)
        #: norm of the gradients, clip factor and whether the step was skipped (1.0), of the last step
        self.stats = self._record[8:20].view(torch.float32)
        eight = state_bits == 8
        self._state = (state_bits, self.m.data_ptr(), self.v.data_ptr(), self.m_scale.data_ptr() if eight else None,
                       self.v_scale.data_ptr() if eight else None)
        self._work = (self._record.data_ptr(), self._scratch.data_ptr(), self._scratch.numel())
        self._hp = B.so_hparams()
        self._written = [*self.params, *(self.copies or ()), self.m, self.v, self._record]
        if state_bits == 8:
            self._written += [self.m_scale, self.v_scale]

    def _check(self, where, what, t, numel):
        if t.device != self.device:
            _refuse(where, f"a {what} is not on the parameters' device")
        if t.numel() != numel or not t.is_contiguous():
            _refuse(where, f"a {what} is not contiguous with its parameter's size")

    def _take_written(self, where):
        """Checks the parameters and copies, and takes their addresses."""
        seen = set()
        for p, numel in zip(self.params, self._numels):
            if p.dtype != torch.float32:
                _refuse(where, "parameters are float32")
            self._check(where, "parameter", p, numel)
            if numel and p.data_ptr() in seen:
                _refuse(where, "a parameter is in the list twice")
            seen.add(p.data_ptr())
        for c, numel in zip(self.copies or (), self._numels):
            if _DTYPES.get(c.dtype) != self._copy_dtype:
                _refuse(where, "there must be a copy for each parameter, all bfloat16 or all float16")
            self._check(where, "copy", c, numel)
        # what is written is written by one warp alone
        end = 0
        both = [*self.params, *(self.copies or ())]
        spans = sorted((t.data_ptr(), t.numel() * t.element_size()) for t in both if t.numel())
        for at, size in spans:
            if at < end:
                _refuse(where, "parameters and copies overlap")
            end = at + size
        self._spans = [at for at, _ in spans], [at + size for at, size in spans]
        for e, p in zip(self._list, self.params):
            e.param = p.data_ptr()
        for e, c in zip(self._list, self.copies or ()):
            e.copy = c.data_ptr()
        self._at_written = both, list(map(_data_ptr, both))
        # an address in use stays its tensor's, also when the tensor has gone elsewhere
        self._held_written = [t.untyped_storage() for t in both]
        self._at_grads = self.grads, None                     # to be compared with these

    def _look(self, where):
        """Parameters and copies that have been given other storage are taken anew."""
        tensors, addresses = self._at_written
        if list(map(_data_ptr, tensors)) != addresses:
            self._take_written(where)

    def set_grads(self, grads: Sequence[torch.Tensor]) -> None:
        """Other gradient tensors from the next step on."""
        self._look("TensorAdamW")
        grads = list(grads)
        dtypes = {g.dtype for g in grads}
        if len(grads) != len(self.params) or len(dtypes) != 1 or not dtypes <= set(_DTYPES):
            _refuse("TensorAdamW", "there must be a gradient for each parameter, all bfloat16, float16 or float32")
        for e, g in zip(self._list, grads):
            self._check("TensorAdamW", "gradient", g, e.numel)
        # gradients are read as what no one writes
        starts, ends = self._spans
        for g in grads:
            if g.numel():
                at = bisect_left(starts, g.data_ptr() + g.numel() * g.element_size())   # (those before begin below its end)
                if at > 0 and ends[at - 1] > g.data_ptr():
                    _refuse("TensorAdamW", "a gradient overlaps a parameter or a copy")
        for e, g in zip(self._list, grads):
            e.grad = g.data_ptr()
        self.grads, self._grad_dtype = grads, _DTYPES[grads[0].dtype]
        self._at_grads = grads, list(map(_data_ptr, grads))
        self._held_grads = [g.untyped_storage() for g in grads]

    def step(self, hp, *, clip: bool = True, grad_scale: float = 1.0, seed: Optional[int] = None, stream=None):
        """One step with the hyper-parameters of `hp` (lr, beta1, beta2, eps,
        weight_decay, max_grad_norm).  `clip` looks at the gradients first: their norm
        is brought down to ``hp.max_grad_norm`` (where that is positive), and a step
        whose norm is not finite is skipped.  `grad_scale` multiplies the gradients (1 /
        loss scale).  `seed` rounds 8-bit moments stochastically.  Returns `stats`.  What is
        given here is a captured step's for all its replays; t and the random numbers go on.

        Runs on the current stream, or on `stream`; the tensors are the optimizer's, which
        the caller keeps until that stream is done with them."""
        where = "tensor_adamw_step"
        if self.device.index != _current_device():
            _refuse(where, "the parameters are not on the current device")
        if seed is not None and self.state_bits != 8:
            _refuse(where, "a seed is for 8-bit moments")
        self._look(where)
        tensors, addresses = self._at_grads
        if list(map(_data_ptr, tensors)) != addresses:
            self.set_grads(tensors)
        h = self._hp
        h.lr, h.beta1, h.beta2, h.eps = hp.lr, hp.beta1, hp.beta2, hp.eps
        h.weight_decay, h.max_grad_norm = hp.weight_decay, hp.max_grad_norm
        status = B.lib().so_tensor_adamw_step(
            self._list, len(self._list), self._grad_dtype, self._copy_dtype, *self._state, C.byref(h), grad_scale, bool(clip),
            seed is not None, (seed or 0) & 0xFFFFFFFFFFFFFFFF, *self._work,
            _raw_stream(self.device.index) if stream is None else stream.cuda_stream)
        if status != B.SO_OK:
            raise B.SuperOffloadError(status, "so_" + where)
        _increment_version(self._written)
        return self.stats

    def moments(self, *, stream=None):
        """(m, v) of all blocks: the fp32 arenas themselves, or bf16 tensors of the values
        that the 8-bit codes stand for, which bf16 holds exactly."""
        if self.state_bits == 32:
            return self.m, self.v
        if self.device.index != _current_device():
            _refuse("tensor_adamw_moments", "the parameters are not on the current device")
        with torch.cuda.stream(stream):
            m, v = (torch.empty(self.m.shape, dtype=torch.bfloat16, device=self.device) for _ in range(2))
            B.so_tensor_adamw_moments(self.m.data_ptr(), self.v.data_ptr(), self.m_scale.data_ptr(),
                                      self.v_scale.data_ptr(), self.blocks, m.data_ptr(), v.data_ptr(),
                                      _raw_stream(self.device.index))
        return m, v

    def block_of(self, index: int) -> int:
        """First block of the index-th tensor in the arenas."""
        return sum(-(-e.numel // B.SO_TENSOR_BLOCK) for e in self._list[:index])

    @property
    def step_count(self) -> int:
        """Steps taken (skipped ones are none); waits for the device."""
        return int(self._record[:8].view(torch.int64).item())

    def set_step(self, t: int) -> None:
        if t < 0:
            _refuse("TensorAdamW", "a step count is not negative")
        self._record[:8].view(torch.int64).fill_(t)

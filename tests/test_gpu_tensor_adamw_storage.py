"""AdamW over a list of tensors whose storage is exchanged underneath (``t.data = other``),
and gradients that lie in what a step writes."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200.tensor_adamw import TensorAdamW
from test_gpu_operators import BF16, gen, randn, same_bits
from test_gpu_tensor_adamw import HP

pytestmark = pytest.mark.gpu
SIZES = [1000, 7, 4096]


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


def make(bits=32):
    g = gen(5)
    params = [torch.nn.Parameter(randn(g, n)) for n in SIZES]
    copies = [p.detach().to(BF16) for p in params]
    grads = [(0.01 * randn(g, n)).to(BF16) for n in SIZES]
    return TensorAdamW(params, grads, copies=copies, state_bits=bits)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("which", ["params", "copies", "grads"])
def test_other_storage_is_taken_up(which, bits):
    """A step after ``t.data = other`` works on the other storage and leaves the old one alone."""
    opt, twin = make(bits), make(bits)
    hp = HP(max_grad_norm=0.5)
    for t in (1, 2):
        old = [x.detach() for x in getattr(opt, which)]               # holds the storage: nobody else gets it
        kept = [x.clone() for x in old]
        for i, x in enumerate(getattr(opt, which)):
            if i != 1 or t == 2:
                x.data = torch.cat([x.detach(), x.detach()])[:x.numel()]
        moved = [a.data_ptr() != x.data_ptr() for a, x in zip(old, getattr(opt, which))]
        assert moved == [True, t == 2, True]
        opt.step(hp)
        twin.step(hp)
        for name in ("params", "copies", "grads"):
            assert all(same_bits(a.detach(), b.detach()) for a, b in zip(getattr(opt, name), getattr(twin, name))), name
        assert same_bits(opt.m, twin.m) and same_bits(opt.v, twin.v)
        assert all(same_bits(a, b) for a, b, gone in zip(old, kept, moved) if gone)


def test_storage_that_does_not_fit_is_refused():
    hp = HP()
    other = {"of another size": lambda x: x.detach()[:500].clone(), "not contiguous": lambda x: x.detach().repeat(2)[::2],
             "empty": lambda x: x.detach()[:0]}
    for what, swap in other.items():
        for which in ("params", "copies", "grads"):
            opt = make()
            t = getattr(opt, which)[0]
            before = [x.detach().clone() for x in (*opt.params, *opt.copies, opt.m, opt.v)]
            right = t.detach()
            t.data = swap(t)
            with pytest.raises(B.SuperOffloadError) as err:
                opt.step(hp)
            assert err.value.status == B.SO_ERR_INVALID_ARG, what
            t.data = right                                # nothing has happened
            assert all(same_bits(a, b.detach()) for a, b in zip(before, (*opt.params, *opt.copies, opt.m, opt.v)))
            assert opt.step_count == 0
            opt.step(hp)
            assert opt.step_count == 1
    opt = make()
    opt.params[2].data = torch.cat([opt.params[0].detach(), opt.params[2].detach()])[:4096]
    opt.params[0].data = opt.params[2].detach()[100:1100]
    with pytest.raises(B.SuperOffloadError, match="overlap"):
        opt.step(hp)


def test_gradients_apart_from_what_is_written():
    arena, low = torch.zeros(2000, device="cuda"), torch.zeros(2000, dtype=BF16, device="cuda")
    p, c = [arena[:300], arena[700:1200]], [low[:300], low[700:1200]]
    apart = [low[300:600], low[1200:1700]]
    for grads in ([arena[:300], arena[1200:1700]],                    # a parameter itself
                  [arena[400:700], arena[299:799]],                   # across a parameter's end and another's start
                  [arena[300:600], arena[1199:1699]]):
        with pytest.raises(B.SuperOffloadError, match="overlap"):
            TensorAdamW(p, grads)
    for grads in ([low[299:599], apart[1]], [apart[0], low[300:800]], [low[100:400], apart[1]]):
        with pytest.raises(B.SuperOffloadError, match="overlap"):
            TensorAdamW(p, grads, copies=c)
        opt = TensorAdamW(p, apart, copies=c)
        with pytest.raises(B.SuperOffloadError, match="overlap"):
            opt.set_grads(grads)
        assert opt.grads[0] is apart[0]
        opt.step(HP())
    # neighbours, an empty tensor anywhere, and gradients in each other are fine
    opt = TensorAdamW([*p, arena[:0]], [arena[300:600], arena[200:700][:0].new_zeros(500), arena[:0]])
    opt.set_grads([arena[1200:1500], arena[1300:1800], arena[100:100]])
    opt.step(HP())


def test_a_parameter_that_moves_into_a_gradient():
    """The step that would take it up is refused, and so is the next one."""
    opt = make()
    opt.set_grads([g.float() for g in opt.grads])
    opt.params[0].data = opt.grads[0]
    for _ in range(2):
        with pytest.raises(B.SuperOffloadError, match="overlap"):
            opt.step(HP())
    assert opt.step_count == 0
    opt.set_grads([torch.zeros_like(opt.grads[0]), *opt.grads[1:]])
    opt.step(HP())

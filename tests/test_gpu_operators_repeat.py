"""Results do not depend on what was called before."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest

from paper_2509_21271_b200 import build as so_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

# Two widths whose kernels are the same and whose shared memory differs by a few hundred
# bytes, on either side of what one more block an SM needs.
PROGRAM = """
import hashlib, sys, torch
from paper_2509_21271_b200 import operators as ops

def gradients(cols):
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, dy = (torch.randn(20000, cols, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    y, mean, rstd = ops.layer_norm_forward(x)
    dx, dw, db = ops.layer_norm_backward(dy, x, mean, rstd, dweight=torch.empty(cols, device="cuda"),
                                         dbias=torch.empty(cols, device="cuda"))
    return b"".join(t.cpu().view(torch.uint8).numpy().tobytes() for t in (y.view(torch.int16), dx.view(torch.int16), dw, db))

for cols in sys.argv[1:]:
    last = gradients(int(cols))
print(hashlib.sha256(last).hexdigest())
"""


def digest(*cols):
    out = subprocess.run([sys.executable, "-c", PROGRAM, *map(str, cols)], capture_output=True, text=True, cwd=ROOT,
                         timeout=300)
    assert out.returncode == 0, out.stderr
    return out.stdout.strip()


@pytest.mark.parametrize("before,cols", [(2320, 2328), (2328, 2320), (3536, 3544), (3544, 3536)])
def test_layer_norm_gradients_do_not_depend_on_the_width_before(before, cols):
    so_build.build_library()
    assert digest(before, cols) == digest(cols)


def test_operators_in_a_torch_graph():
    """From a Function they take part in autograd; what they overwrite is noticed by a graph
    that saved it."""
    import torch

    from paper_2509_21271_b200 import binding as B
    from paper_2509_21271_b200 import operators as ops

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, mean, rstd = ops.layer_norm_forward(x, w, b)
            ctx.save_for_backward(x, w, mean, rstd)
            return y

        @staticmethod
        def backward(ctx, dy):
            x, w, mean, rstd = ctx.saved_tensors
            return ops.layer_norm_backward(dy.contiguous(), x, mean, rstd, w)

    so_build.build_library()
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, b, v = (torch.randn(s, generator=g, device="cuda") for s in ((40, 96), (96,), (96,), (40, 96)))
    for t in (x, w, b):
        t.requires_grad_()
    with pytest.raises(B.SuperOffloadError, match="requires grad"):
        ops.layer_norm_forward(x, w, b)
    got = torch.autograd.grad((Norm.apply(x, w, b) * v).sum(), (x, w, b))
    want = torch.autograd.grad((torch.nn.functional.layer_norm(x.double(), (96,), w.double(), b.double()) * v).sum(), (x, w, b))
    for p, q in zip(got, want):
        # fp32 throughout: sums of at most 96 terms, roundings of 2^-24 each
        assert (p - q).abs().max() <= 200 * 2.0 ** -24 * q.abs().max()

    logits = torch.randn(8, 50, generator=g, device="cuda", requires_grad=True)
    ids, teacher = torch.zeros(8, 1, dtype=torch.int64, device="cuda"), torch.zeros(8, 1, device="cuda")
    for overwrite in (lambda t: ops.distill_loss(t, ids, teacher, grad=t),
                      lambda t: ops.policy_loss(t, ids[:, 0].contiguous(), teacher[:, 0].contiguous(), grad=t),
                      lambda t: ops.layer_norm_forward(t, out=t),
                      lambda t: ops.layer_norm_backward(t, t.clone(), teacher[:, 0].contiguous(), teacher[:, 0].contiguous(), dx=t),
                      lambda t: ops.embedding_backward(ids[:, 0].contiguous(), t.clone(), t)):
        z = logits.exp()                          # exp saves its result
        with torch.no_grad():
            overwrite(z)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.sum().backward()

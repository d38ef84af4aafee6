"""The operators and the optimizer together: the example's student against autograd
in fp32, and a few steps of training with either loss."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest
import torch

from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200 import operators as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    so_build.build_library()
    torch.cuda.set_device(0)
    import train_student
    return train_student


def test_gradients_of_a_step_against_autograd(example):
    """bf16 activations and gradients against fp32 autograd through the same formulas:
    the roundings (2^-8 each) of some ten operators in a row, random in sign, stay well
    below 8 % of each gradient's norm."""
    student = example.Student(vocab=1003, width=96, blocks=2)
    ids = torch.randint(40, (130,), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    teacher_ids, teacher_logits = example.teacher_lists(1003, 6)
    logits, state = student.forward(ids)
    weight = torch.full((130,), 1 / 130, device="cuda")
    loss, _, dlogits = ops.distill_loss(logits, teacher_ids[ids], teacher_logits[ids], weight)
    student.backward(dlogits, state)

    p = {k: v.float().requires_grad_() for k, v in student.param.items()}
    h = p["table"][ids] * (96 ** 0.5 * 0.1)
    norm = lambda x, n: torch.nn.functional.layer_norm(x, (96,), p[n + ".w"], p[n + ".b"])  # noqa: E731
    for i in range(2):
        h = h + torch.relu(norm(h, f"norm{i}") @ p[f"up{i}"]).square() @ p[f"down{i}"]
    logq = torch.log_softmax(norm(h, "norm") @ p["table"].t(), 1)
    logp = torch.log_softmax(teacher_logits[ids], 1)
    want = (logp.exp() * (logp - logq.gather(1, teacher_ids[ids].long()))).sum(1).mean()
    want.backward()
    assert abs(loss.item() - want.item()) <= 0.02 * abs(want.item())
    for name, g in student.grad.items():
        ref = p[name].grad
        assert (g.float() - ref).norm().item() <= 0.08 * ref.norm().item(), name


def test_distillation_lowers_the_loss(example):
    losses, decisions = example.train(steps=40)
    assert all(x == x for x in losses)
    assert sum(losses[-5:]) < 0.6 * sum(losses[:5])
    assert set(decisions) <= {0, 2}                  # kept, or stepped again with clipped gradients


def test_policy_raises_the_advantage(example):
    values, decisions = example.train(steps=60, policy=True)
    assert sum(values[-10:]) > sum(values[:10])
    assert set(decisions) <= {0, 2}


def test_a_nan_in_the_loss_skips_the_step(example):
    student = example.Student(vocab=1003, width=64, blocks=1)
    before = [t.clone() for t in student.opt.gather_state()]
    ids = torch.arange(32, device="cuda")
    logits, state = student.forward(ids)
    logits[3, 17] = float("nan")
    loss, _, dlogits = ops.distill_loss(logits, ids[:, None], torch.zeros(32, 1, device="cuda"))
    assert torch.isnan(loss).all()
    student.backward(dlogits, state)
    result = student.step(example.HParams())
    assert result.decision == 1 and result.step_after == 0
    assert all(torch.equal(a, b) for a, b in zip(before, student.opt.gather_state()))


def test_example_runs_as_a_program(example):
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "train_student.py"), "--steps", "3"],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    assert len(out.stdout.strip().splitlines()) == 3

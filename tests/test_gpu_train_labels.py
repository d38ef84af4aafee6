"""The loss from the hidden states, the norms on both sides of residuals and AdamW over a
list of tensors in one training step: the example's student of labels against autograd in
fp32, and its step captured and replayed."""
from __future__ import annotations

import os
import subprocess
import sys

import pytest
import torch

from paper_2509_21271_b200 import build as so_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    so_build.build_library()
    torch.cuda.set_device(0)
    import train_student
    return train_student


def batch(vocab, tokens, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(40, (tokens,), generator=g, device="cuda")
    labels = torch.randint(vocab, (tokens,), generator=g, device="cuda")
    labels[::5] = -100
    weight = torch.rand(tokens, generator=g, device="cuda") / tokens
    weight[::7] = 0.0
    return ids, labels, weight


@pytest.mark.parametrize("tokens,vocab,width", [(130, 1003, 96), (300, 2000, 128)])
def test_gradients_of_a_step_against_autograd(example, tokens, vocab, width):
    """bf16 activations and gradients against fp32 autograd through the same formulas:
    the roundings (2^-8 each) of some ten operators in a row, random in sign, stay well
    below 8 % of each gradient's norm."""
    student = example.LabelStudent(vocab=vocab, width=width)
    ids, labels, weight = batch(vocab, tokens)
    loss = student.loss_and_gradients(ids, labels, weight)
    p = {k: v.float().requires_grad_() for k, v in student.param.items()}
    rms = lambda x: x * (x.square().mean(1, keepdim=True) + 1e-5).rsqrt()  # noqa: E731
    h = p["table"][ids] * width ** 0.5
    x = torch.nn.functional.layer_norm(h, (width,), p["norm.w"], p["norm.b"])
    for i in range(2):
        block = torch.relu(x @ p[f"up{i}"]).square() @ p[f"down{i}"]
        h = h + p[f"gate{i}"] * (rms(block) * p[f"post{i}"])
        x = rms(h) * p[f"pre{i}"]
    live = (labels >= 0) & (weight != 0)
    logp = torch.log_softmax(x @ p["table"].t(), 1)
    want = -(weight * logp.gather(1, labels.clamp(min=0)[:, None])[:, 0])[live].sum()
    want.backward()
    assert abs(loss.item() - want.item()) <= 0.02 * abs(want.item())
    for name, g in student.grad.items():
        ref = p[name].grad
        assert (g.float() - ref).norm().item() <= 0.08 * ref.norm().item(), name


@pytest.mark.parametrize("state_bits", [8, 32])
def test_a_whole_step_captured_and_replayed(example, state_bits):
    """Graph replays take the same steps as eager calls, bit for bit."""
    hp = example.HParams()
    eager, replayed = (example.LabelStudent(vocab=1003, width=128, state_bits=state_bits) for _ in range(2))
    ids, labels, weight = batch(1003, 200)
    replayed.loss_and_gradients(ids, labels, weight)      # libraries set themselves up outside of the capture
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            loss = replayed.loss_and_gradients(ids, labels, weight)
            replayed.step(hp)
    torch.cuda.current_stream().wait_stream(side)
    for seed in (6, 7, 8):
        for t, new in zip((ids, labels, weight), batch(1003, 200, seed)):
            t.copy_(new)
        graph.replay()
        want = eager.loss_and_gradients(ids, labels, weight)
        eager.step(hp)
        assert torch.equal(loss, want)
        for name, m in eager.master.items():
            assert torch.equal(m, replayed.master[name]) and torch.equal(eager.param[name], replayed.param[name]), name
        assert torch.equal(eager.opt.m, replayed.opt.m) and torch.equal(eager.opt.v, replayed.opt.v)
    assert eager.opt.step_count == replayed.opt.step_count == 3


def test_a_nan_skips_the_step(example):
    student = example.LabelStudent(vocab=1003, width=64, blocks=1)
    ids, labels, weight = batch(1003, 64)
    student.param["up0"][3, 5] = float("nan")
    before = [t.clone() for t in (*student.master.values(), student.opt.m, student.opt.v)]
    assert torch.isnan(student.loss_and_gradients(ids, labels, weight)).all()
    assert student.step(example.HParams())[2].item() == 1.0 and student.opt.step_count == 0
    assert all(torch.equal(a, b) for a, b in zip(before, (*student.master.values(), student.opt.m, student.opt.v)))


def test_example_runs_as_a_program(example):
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "train_student.py"), "--steps", "3", "--labels"],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    lines = out.stdout.strip().splitlines()
    assert len(lines) == 3 and all(line.endswith("STEP") for line in lines)

"""A small student trained with the operators around the matrix products and the
bucketed speculative AdamW step behind them.

The student is an embedding, a few residual blocks (layer norm, up-projection,
ReLU squared, down-projection), a final layer norm and a head that shares the
embedding's table.  Its loss is distillation from a fixed teacher's top logits, or
with ``--policy`` the clipped policy loss on tokens sampled from the student.
Activations are bf16; every parameter's gradient is written straight into the
optimizer's bf16 gradient arena, the table's in two parts: the head's matrix
product writes it, the embedding's backward pass adds to it.

With ``--labels`` another student learns the next token from labels: RMS norms on both
sides of every residual with a learned gate, the cross entropy and both gradients of the
head straight from the hidden states, and parameters in tensors of their own under AdamW
with 8-bit moments.

    python examples/train_student.py --steps 40
    python examples/train_student.py --steps 40 --policy
    python examples/train_student.py --steps 40 --labels
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2509_21271_b200 import binding as B                      # noqa: E402
from paper_2509_21271_b200 import operators as ops                  # noqa: E402
from paper_2509_21271_b200.optimizer import BucketedAdamW           # noqa: E402
from paper_2509_21271_b200.tensor_adamw import TensorAdamW          # noqa: E402


@dataclass
class HParams:
    lr: float = 3e-3
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    weight_decay: float = 0.01
    max_grad_norm: float = 1.0


class Student:
    """Parameters, their gradients, and one training step by hand."""

    def __init__(self, vocab: int = 4001, width: int = 256, blocks: int = 2, seed: int = 0):
        self.vocab, self.width, self.blocks = vocab, width, blocks
        shapes = [("table", (vocab, width))]
        for i in range(blocks):
            shapes += [(f"norm{i}.w", (width,)), (f"norm{i}.b", (width,)), (f"up{i}", (width, 4 * width)),
                       (f"down{i}", (4 * width, width))]
        shapes += [("norm.w", (width,)), ("norm.b", (width,))]
        numel = [torch.Size(s).numel() for _, s in shapes]
        # buckets of a multiple of 64 elements: arenas are flat, tensors are views of them
        self.opt = BucketedAdamW(numel, bucket_elems=max(64, sum(numel) // 3 // 64 * 64))
        self.param, self.grad = {}, {}
        gen = torch.Generator(device="cuda").manual_seed(seed)
        start, flat = 0, torch.empty(sum(numel), device="cuda")
        for (name, shape), n in zip(shapes, numel):
            self.param[name] = self.opt.param_bf16[start:start + n].view(shape)
            self.grad[name] = self.opt.grad[start:start + n].view(shape)
            init = torch.ones(n, device="cuda") if name.endswith(".w") else torch.zeros(n, device="cuda") \
                if name.endswith(".b") else torch.randn(n, generator=gen, device="cuda") * shape[0] ** -0.5
            flat[start:start + n] = init if name != "table" else init * (vocab ** 0.5) * 0.1
            start += n
        self.opt.load_state(flat)
        self.opt.cast_params(stream=torch.cuda.current_stream())

    def forward(self, ids):
        """(logits, what the backward pass needs)."""
        p, kept = self.param, []
        h = ops.embedding_forward(ids, p["table"], self.width ** 0.5 * 0.1)
        for i in range(self.blocks):
            x, mean, rstd = ops.layer_norm_forward(h, p[f"norm{i}.w"], p[f"norm{i}.b"])
            up = torch.matmul(x, p[f"up{i}"])
            act = torch.relu(up).square_()
            kept.append((h, x, mean, rstd, up, act))
            h = h + torch.matmul(act, p[f"down{i}"])
        x, mean, rstd = ops.layer_norm_forward(h, p["norm.w"], p["norm.b"])
        return torch.matmul(x, p["table"].t()), (ids, kept, h, x, mean, rstd)

    def backward(self, dlogits, state):
        """Gradients of all parameters into the arena."""
        p, g = self.param, self.grad
        ids, kept, h, x, mean, rstd = state
        torch.mm(dlogits.t(), x, out=g["table"])
        dh, _, _ = ops.layer_norm_backward(torch.matmul(dlogits, p["table"]), h, mean, rstd, p["norm.w"],
                                           dweight=g["norm.w"], dbias=g["norm.b"])
        for i in reversed(range(self.blocks)):
            h, x, mean, rstd, up, act = kept[i]
            torch.mm(act.t(), dh, out=g[f"down{i}"])
            dup = torch.matmul(dh, p[f"down{i}"].t()).mul_(torch.relu(up).mul_(2.0))
            torch.mm(x.t(), dup, out=g[f"up{i}"])
            dx, _, _ = ops.layer_norm_backward(torch.matmul(dup, p[f"up{i}"].t()), h, mean, rstd, p[f"norm{i}.w"],
                                               dweight=g[f"norm{i}.w"], dbias=g[f"norm{i}.b"])
            dh = dh + dx
        ops.embedding_backward(ids, dh, g["table"], self.width ** 0.5 * 0.1, accumulate=True)

    def step(self, hp: HParams):
        return self.opt.iteration(hp, stream=torch.cuda.current_stream())


class LabelStudent:
    """A student of labels: parameters, gradients and bf16 copies in tensors of their own."""

    def __init__(self, vocab: int = 4001, width: int = 256, blocks: int = 2, seed: int = 0, state_bits: int = 8):
        self.vocab, self.width, self.blocks = vocab, width, blocks
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        one = lambda at: torch.full((width,), at, device="cuda")  # noqa: E731
        self.master = {"table": rand(vocab, width) * width ** -0.5, "norm.w": one(1.0), "norm.b": one(0.0)}
        for i in range(blocks):
            self.master.update({f"up{i}": rand(width, 4 * width) * width ** -0.5, f"gate{i}": one(0.5), f"post{i}": one(1.0),
                                f"down{i}": rand(4 * width, width) * (4 * width) ** -0.5, f"pre{i}": one(1.0)})
        self.param = {k: v.to(torch.bfloat16) for k, v in self.master.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in self.param.items()}
        self.opt = TensorAdamW(list(self.master.values()), list(self.grad.values()), copies=list(self.param.values()),
                               state_bits=state_bits)

    def forward(self, ids):
        """(hidden states, what the backward pass needs)."""
        p, kept = self.param, []
        h = ops.embedding_forward(ids, p["table"], self.width ** 0.5)
        x, mean, rstd = ops.layer_norm_forward(h, p["norm.w"], p["norm.b"])
        first = (h, mean, rstd)
        for i in range(self.blocks):
            up = torch.matmul(x, p[f"up{i}"])
            act = torch.relu(up).square_()
            block = torch.matmul(act, p[f"down{i}"])
            before = x
            h, x, stats = ops.residual_norm_forward(h, block, p[f"gate{i}"], p[f"post{i}"], None, p[f"pre{i}"], None,
                                                    kind="rms")
            kept.append((before, up, act, block, h, stats))
        return x, (ids, first, kept)

    def loss_and_gradients(self, ids, labels, weight):
        """The loss; the gradients of all parameters."""
        p, g = self.param, self.grad
        hidden, (ids, first, kept) = self.forward(ids)
        loss, _, dx, _ = ops.linear_cross_entropy(hidden, p["table"], labels, weight, dtable=g["table"])
        dh = None
        for i in reversed(range(self.blocks)):
            before, up, act, block, h, stats = kept[i]
            dh, dblock, *_ = ops.residual_norm_backward(
                dx, dh, h, block, stats, p[f"gate{i}"], p[f"post{i}"], None, p[f"pre{i}"], kind="rms", dgate=g[f"gate{i}"],
                dpost_weight=g[f"post{i}"], dweight=g[f"pre{i}"])
            torch.mm(act.t(), dblock, out=g[f"down{i}"])
            dup = torch.matmul(dblock, p[f"down{i}"].t()).mul_(torch.relu(up).mul_(2.0))
            torch.mm(before.t(), dup, out=g[f"up{i}"])
            dx = torch.matmul(dup, p[f"up{i}"].t())
        h, mean, rstd = first
        dx, _, _ = ops.layer_norm_backward(dx, h, mean, rstd, p["norm.w"], dweight=g["norm.w"], dbias=g["norm.b"])
        ops.embedding_backward(ids, dx if dh is None else dx + dh, g["table"], self.width ** 0.5, accumulate=True)
        return loss

    def step(self, hp: HParams, seed: int | None = 0):
        return self.opt.step(hp, seed=seed if self.opt.state_bits == 8 else None)


def train_labels(steps: int = 40, tokens: int = 512, student: LabelStudent | None = None, hp=None):
    """Losses by step, and whether each was skipped: the next token is a fixed function of the last."""
    student, hp = student or LabelStudent(), hp or HParams()
    gen = torch.Generator(device="cuda").manual_seed(3)
    follows = torch.randint(student.vocab, (student.vocab,), generator=gen, device="cuda")
    losses, skipped = [], []
    for _ in range(steps):
        ids = torch.randint(64, (tokens,), generator=gen, device="cuda")
        labels = follows[ids]
        labels[::8] = -100                            # as where a prompt is not learned
        weight = (labels >= 0) / (labels >= 0).sum()
        losses.append(student.loss_and_gradients(ids, labels, weight)[0])
        skipped.append(student.step(hp)[2].clone())
    return [float(x) for x in losses], [bool(x) for x in skipped]


def teacher_lists(vocab: int, top_k: int, seed: int = 1):
    """A fixed teacher: for each token the ids that may follow, and their logits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(vocab, (vocab, top_k), generator=gen, device="cuda", dtype=torch.int32)
    return ids, torch.randn(vocab, top_k, generator=gen, device="cuda") * 1.5


def train(steps: int = 40, tokens: int = 512, policy: bool = False, student: Student | None = None, hp=None):
    """Losses by step; prints nothing."""
    student, hp = student or Student(), hp or HParams()
    gen = torch.Generator(device="cuda").manual_seed(3)
    teacher_ids, teacher_logits = teacher_lists(student.vocab, 8)
    losses, decisions = [], []
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    for _ in range(steps):
        ids = torch.randint(64, (tokens,), generator=gen, device="cuda")
        logits, state = student.forward(ids)
        if policy:
            # tokens sampled from the student; the teacher's list decides what is good
            chosen = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=gen)[:, 0]
            liked = (teacher_ids[ids] % 7 == chosen[:, None] % 7).any(1)
            advantage = torch.where(liked, 1.0, -1.0)
            # the gradient takes the logits' place: they are not needed any more
            loss, _, _, dlogits = ops.policy_loss(logits, chosen, advantage, weight, grad=logits)
            losses.append(advantage.mean())
        else:
            loss, _, dlogits = ops.distill_loss(logits, teacher_ids[ids], teacher_logits[ids], weight, grad=logits)
            losses.append(loss[0])
        student.backward(dlogits, state)
        decisions.append(student.step(hp).decision)
    return [float(x) for x in losses], decisions


def main():
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=40)
    parser.add_argument("--tokens", type=int, default=512)
    parser.add_argument("--policy", action="store_true")
    parser.add_argument("--labels", action="store_true")
    args = parser.parse_args()
    if args.labels:
        for i, (v, gone) in enumerate(zip(*train_labels(args.steps, args.tokens)), 1):
            print(f"step {i:3d}  loss {v:8.4f}  {'SKIP' if gone else 'STEP'}")
        return
    values, decisions = train(args.steps, args.tokens, args.policy)
    what = "mean advantage" if args.policy else "loss"
    for i, (v, d) in enumerate(zip(values, decisions), 1):
        print(f"step {i:3d}  {what} {v:8.4f}  {B.DECISION_NAMES[d]}")


if __name__ == "__main__":
    main()

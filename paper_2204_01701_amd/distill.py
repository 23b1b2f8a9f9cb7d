"""A quadratic classifier distilled from a first-order teacher, on synthetic data.

The student is the kind of network the paper's library trains (arXiv 2204.01701, section 4.2:
quadratic layers with a ReLU, first-order layers beside them): a quadratic fully-connected layer,
a first-order block with activation and residual, a linear classifier.  The teacher is first-order
and wider.  One step, all of it in the library's kernels but the update:

* the teacher's logits (``linear_act``) and, of those, the most likely classes (``token_logprobs``);
* the student's logits (``quad_linear``, ``linear_act``);
* the loss against the teacher's places and the label (``distill_loss``) and its gradient, back
  through every layer;
* plain gradient descent on float32 master weights.

``evaluate`` scores the labels of held-out rows: their log probability, the entropy of the answers
and how often the best class is the label's and the teacher's.

Usage: ``python -m paper_2204_01701_amd.distill [--steps 60] [--classes 200] [--dtype bf16]``.
"""
from __future__ import annotations

import argparse
import math

import torch

from .autograd import distill_loss, linear_act, quad_linear, token_logprobs

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


class Data:
    """Rows scattered around one centre per class, in `width` dimensions."""

    def __init__(self, classes, width, seed, device):
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.device = device
        self.centre = torch.randn(classes, width, generator=self.gen, device=device)

    def batch(self, rows, dtype):
        label = torch.randint(len(self.centre), (rows,), generator=self.gen, device=self.device)
        noise = torch.randn(rows, self.centre.shape[1], generator=self.gen, device=self.device)
        return (self.centre[label] + 0.8 * noise).to(dtype), label


class Teacher:
    """A first-order network whose classifier knows the centres: logits of cosine-like scores through one gelu block."""

    def __init__(self, data, dtype):
        classes, width = data.centre.shape
        self.mix = (torch.randn(width, width, generator=data.gen, device=data.device) * (0.1 / math.sqrt(width))).to(dtype)
        self.head = (data.centre * (4.0 / math.sqrt(width))).to(dtype)
        self.bias = torch.zeros(classes, device=data.device)

    @torch.no_grad()
    def top(self, x, k, label):
        """The k most likely classes, their log probabilities and the labels'."""
        z = linear_act(linear_act(x, self.mix, act="gelu", residual=x), self.head, self.bias)
        logp, _, top_logp, top_ids = token_logprobs(z, label, top=k)
        return top_ids, top_logp, logp


class Student:
    """quadratic layer (ReLU) -> first-order block with silu and residual -> classifier, float32 master weights."""

    def __init__(self, width, hidden, classes, dtype, device, seed):
        gen = torch.Generator(device=device).manual_seed(seed)

        def weight(out, inp, scale=1.0):
            return (torch.randn(out, inp, generator=gen, device=device) * (scale / math.sqrt(inp))).requires_grad_(True)

        def bias(out, value=0.0):
            return torch.full((out,), value, device=device).requires_grad_(True)

        self.dtype = dtype
        self.quad_w = [weight(hidden, width) for _ in range(3)]
        self.quad_b = [bias(hidden, v) for v in (0.0, 0.5, 0.0)]
        self.block_w, self.block_b = weight(hidden, hidden, 0.5), bias(hidden)
        self.head_w, self.head_b = weight(classes, hidden), bias(classes)
        self.weights = [*self.quad_w, *self.quad_b, self.block_w, self.block_b, self.head_w, self.head_b]

    def logits(self, x):
        h = quad_linear(x, *(w.to(self.dtype) for w in self.quad_w), *self.quad_b, relu=True)
        h = linear_act(h, self.block_w.to(self.dtype), self.block_b, residual=h, act="silu")
        return linear_act(h, self.head_w.to(self.dtype), self.head_b)

    @torch.no_grad()
    def update(self, grads, rate):
        # (a clipped step: the quadratic layer's gradients grow with its inputs' squares)
        norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
        scale = rate / norm.clamp_min(1.0)
        for w, g in zip(self.weights, grads):
            w -= scale * g


def train_step(student, teacher, x, label, top, temperature, alpha, rate):
    """One step of distillation; returns the batch's mean loss (on the GPU)."""
    ids, logits, _ = teacher.top(x, top, label)
    loss = distill_loss(student.logits(x), ids, logits, label, temperature=temperature, alpha=alpha).mean()
    student.update(torch.autograd.grad(loss, student.weights), rate)
    return loss.detach()


@torch.no_grad()
def evaluate(student, teacher, x, label):
    """Mean log probability of the labels, mean entropy, and the shares of rows whose best class is the label's and
    the teacher's."""
    logp, entropy, _, best = token_logprobs(student.logits(x), label, top=1)
    theirs, _, _ = teacher.top(x, 1, label)
    return {"logp": logp.mean().item(), "entropy": entropy.mean().item(),
            "accuracy": (best[:, 0] == label).float().mean().item(), "agreement": (best == theirs).float().mean().item()}


def run(steps=60, rows=512, classes=200, width=128, hidden=256, top=20, temperature=2.0, alpha=0.7, rate=0.5, dtype="bf16",
        seed=0, device="cuda:0", report=None):
    """Trains a student; returns (losses of the steps, evaluation before, evaluation after)."""
    dt = DTYPES[dtype]
    data = Data(classes, width, seed, device)
    teacher = Teacher(data, dt)
    student = Student(width, hidden, classes, dt, device, seed + 1)
    held = data.batch(4 * rows, dt)
    before = evaluate(student, teacher, *held)
    losses = []
    for step in range(steps):
        losses.append(train_step(student, teacher, *data.batch(rows, dt), top, temperature, alpha, rate))
        if report and (step % 10 == 0 or step == steps - 1):
            report(step, losses[-1].item())
    return [v.item() for v in losses], before, evaluate(student, teacher, *held)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--classes", type=int, default=200)
    ap.add_argument("--top", type=int, default=20)
    ap.add_argument("--dtype", choices=sorted(DTYPES), default="bf16")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    _, before, after = run(a.steps, a.rows, a.classes, top=a.top, dtype=a.dtype, seed=a.seed,
                           report=lambda step, loss: print(f"step {step:4d}  loss {loss:.4f}", flush=True))
    for name, v in (("before", before), ("after", after)):
        print(f"{name:>6}: " + "  ".join(f"{k} {x:.4f}" for k, x in v.items()))


if __name__ == "__main__":
    main()

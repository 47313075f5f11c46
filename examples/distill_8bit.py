"""A student whose layers keep their weights in 8-bit integers, fitted to a teacher that tells only its largest logits:

  gated block (i8.gated, i8.linear) -> head over the vocabulary (i8.linear) -> divergence of the teacher's top logits from the student's
  softmax, with its gradient (distill.loss_and_gradient) -> the layers' gradients (i8.linear_backward, i8.gated_backward) -> Muon's step on
  the float32 master weights (muon.step) -> 8-bit weights again.

    python examples/distill_8bit.py [--steps 60]

The task is synthetic: the teacher is a fixed random network of the same shape in float32, and the student sees the same four batches over
and over.  Prints the loss every ten steps.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1811_03617_amd import distill, i8, muon  # noqa: E402

DEV = "cuda:0"
WIDTH, HIDDEN, VOCAB = 256, 512, 2000
TOP = 32                          # logits that the teacher tells
TEMPERATURE = 2.0


class Layer:
    """Float32 master weight, its momentum, and the weight in 8 bits, a scale for each row of it and of its transpose."""

    def __init__(self, n_in, n_out, gen):
        self.weight = torch.randn(n_out, n_in, generator=gen, device=DEV) / n_in ** 0.5
        self.buffer = torch.zeros_like(self.weight)
        self.pack()

    def pack(self):
        self.q, self.qt = i8.quantize_both(self.weight)


def network(gen):
    """[gate | up], down, head."""
    return [Layer(WIDTH, 2 * HIDDEN, gen), Layer(HIDDEN, WIDTH, gen), Layer(WIDTH, VOCAB, gen)]


def tell(teacher, x):
    """The teacher's largest logits and where they are, from its float32 weights."""
    both, down, head = (layer.weight for layer in teacher)
    g, u = (x.float() @ both.t()).chunk(2, 1)
    logits = ((torch.nn.functional.silu(g) * u) @ down.t()) @ head.t()
    return logits.topk(TOP, 1)


def gradients(student, x, top, index, weight):
    """Every token's loss, and the gradients of the sum of them by the three weights."""
    both, down, head = student
    h = i8.gated(x, both.q)
    y = i8.linear(h, down.q)
    losses, dz = distill.loss_and_gradient(i8.linear(y, head.q), top, index, temperature=TEMPERATURE, weight=weight)
    dy, d_head = i8.linear_backward(dz, y, head.qt)
    dh, d_down = i8.linear_backward(dy, h, down.qt)
    _, d_both = i8.gated_backward(dh, x, both.q, None, need_dx=False)
    return losses, [d_both, d_down, d_head]


def train(steps=60, batch=512, seed=0, tell_loss=print):
    """Losses of all steps."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    teacher, student = network(gen), network(gen)
    batches = [torch.randn(batch, WIDTH, generator=gen, device=DEV).bfloat16() for _ in range(4)]
    told = [tell(teacher, x) for x in batches]
    weight = torch.full((batch,), 1.0 / batch, device=DEV)
    losses = []
    for step in range(steps):
        at = step % len(batches)
        parts, grads = gradients(student, batches[at], *told[at], weight)
        for layer, grad in zip(student, grads):
            muon.step(layer.weight, grad, layer.buffer, lr=0.03)
            layer.pack()
        losses.append(parts.sum().item())
        if step % 10 == 0:
            tell_loss(f"step {step:4d}  loss {losses[-1]:.4f}")
    tell_loss(f"step {steps - 1:4d}  loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    train(ap.parse_args().steps)

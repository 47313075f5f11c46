"""A small network trained by simulated data-parallel workers, every part through the library:

  4-bit weights (mx.quantize_both) -> forward and backward products on them (mx.linear, mx.linear_backward, output gradients rounded
  stochastically) -> every worker's gradient compressed, the compressed vectors summed, the sum decompressed (gvq.Basis) ->
  Muon's step on the float32 master weights (muon.step) -> 4-bit weights again.

    python examples/train_compressed.py [--steps 60] [--workers 4] [--uncompressed]

The task is synthetic: recover the targets of a fixed random network of the same shape.  Prints the loss every ten steps and the
share of the gradient's numbers that the workers exchange.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1811_03617_amd import gvq, muon, mx  # noqa: E402

DEV = "cuda:0"
SIZES = [256, 512, 512, 128]      # features into and out of each layer
D, K = 128, 32                    # the codec's slice and how many components of it are kept
FIT = 8                           # aggregated gradients a basis is fitted on, exchanged as they are
REFIT = 40                        # steps that a basis serves


class Layer:
    """Float32 master weight, its momentum, and the weight in 4 bits along both axes."""

    def __init__(self, n_in, n_out, gen):
        self.weight = torch.randn(n_out, n_in, generator=gen, device=DEV) / n_in ** 0.5
        self.buffer = torch.zeros_like(self.weight)
        self.pack()

    def pack(self):
        self.q, self.qt = mx.quantize_both(self.weight)


def forward(layers, x):
    """Inputs of every layer, and the last one's outputs."""
    inputs = []
    for i, layer in enumerate(layers):
        inputs.append(x)
        x = mx.linear(x, layer.q)
        if i + 1 < len(layers):
            x = torch.relu(x)
    return inputs, x


def gradient(layers, x, target, gen):
    """One worker's gradient, flattened layer by layer, and its loss."""
    inputs, y = forward(layers, x)
    diff = y.float() - target
    loss = diff.square().mean()
    dy = (2.0 / diff.numel() * diff).to(x.dtype)
    parts = [None] * len(layers)
    for i in reversed(range(len(layers))):
        noise = torch.randint(0, 256, dy.shape, generator=gen, device=DEV, dtype=torch.uint8)
        dx, parts[i] = mx.linear_backward(dy, inputs[i], layers[i].qt, noise=noise, need_dx=i > 0)
        if i > 0:
            dy = dx * (inputs[i] > 0)
    return torch.cat([p.reshape(-1) for p in parts]), loss


class Exchange:
    """Sum of the workers' gradients through the codec: the first FIT of every REFIT steps as they are, to fit the basis on."""

    def __init__(self, n, workers, compressed):
        self.workers, self.compressed, self.step, self.fit = workers, compressed, 0, []
        self.basis = gvq.Basis(n, D, K)
        self.comps = [torch.empty(self.basis.S * K, device=DEV) for _ in range(workers)]
        self.total = torch.empty(self.basis.S * K, device=DEV)
        self.numbers = 0

    def sum(self, grads):
        at = self.step % REFIT
        self.step += 1
        if at < FIT or not self.compressed:
            total = torch.stack(grads).sum(0)
            if self.compressed:
                self.fit.append(total)
                if len(self.fit) == FIT:
                    self.basis.fit(self.fit)
                    self.fit = []
            self.numbers += total.numel()
            return total
        for g, c in zip(grads, self.comps):
            self.basis.compress(g, self.workers, c)
        self.basis.aggregate(self.comps, self.total)
        out = torch.empty_like(grads[0])
        self.basis.decompress(self.total, out)
        self.numbers += self.total.numel()
        return out


def train(steps=60, workers=4, batch=256, compressed=True, seed=0, tell=print):
    """Losses of all steps, and the share of the gradient's numbers that went over the wire."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    teacher = [Layer(a, b, gen) for a, b in zip(SIZES[:-1], SIZES[1:])]
    layers = [Layer(a, b, gen) for a, b in zip(SIZES[:-1], SIZES[1:])]
    n = sum(layer.weight.numel() for layer in layers)
    exchange = Exchange(n, workers, compressed)
    losses = []
    for step in range(steps):
        grads, loss = [], 0.0
        for _ in range(workers):
            x = torch.randn(batch, SIZES[0], generator=gen, device=DEV).bfloat16()
            target = forward(teacher, x)[1].float()
            g, part = gradient(layers, x, target, gen)
            grads.append(g)
            loss = loss + part / workers
        total = exchange.sum(grads) / workers
        at = 0
        for layer in layers:
            count = layer.weight.numel()
            muon.step(layer.weight, total[at:at + count].view_as(layer.weight), layer.buffer, lr=0.02)
            layer.pack()
            at += count
        losses.append(loss.item())
        if step % 10 == 0:
            tell(f"step {step:4d}  loss {losses[-1]:.4f}")
    share = exchange.numbers / (n * steps)
    tell(f"step {steps - 1:4d}  loss {losses[-1]:.4f}  numbers exchanged: {100 * share:.0f} % of the gradients'")
    return losses, share


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--uncompressed", action="store_true")
    a = ap.parse_args()
    train(a.steps, a.workers, compressed=not a.uncompressed)

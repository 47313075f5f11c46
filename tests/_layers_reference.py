"""Plain forms of the 8-bit layers, the gated block and the loss on a teacher's top logits, in numpy float64 (test infrastructure: nothing
here uses the library)."""
import math

import numpy as np

SMALLEST = np.float32(2.0 ** -100)
F32_HALF = 2.0 ** -24            # half a step, relative to the value
BF16_HALF = 2.0 ** -8


def integers(x):
    """(codes as int64, scales float32, which rows are numbers) of the rows of x: the definition, step by step."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(1) if x.shape[1] else np.zeros(x.shape[0], np.float32)
    fine = np.isfinite(top)
    m = np.maximum(np.where(fine, top, 1), SMALLEST).astype(np.float32)
    up, down = np.float32(127) / m, m / np.float32(127)
    # both factors have 24 bits: their product is exact in float64
    q = np.rint(np.where(fine[:, None], x, 0).astype(np.float64) * up.astype(np.float64)[:, None]).astype(np.int64)
    return q, np.where(fine, down, np.float32("nan")).astype(np.float32), fine


def product(a, b):
    """A B^T of two results of `integers`: the sum exact, one rounding to float32, one of the scales' product, one of theirs."""
    sums = (a[0] @ b[0].T).astype(np.float32)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        return (sums * (a[1][:, None] * b[1][None, :])).astype(np.float32)


def values(a):
    return a[0].astype(np.float64) * a[1].astype(np.float64)[:, None]


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activation(g, kind):
    """act(g) and its derivative."""
    g = np.asarray(g, np.float64)
    if kind == "silu":
        s = 1 / (1 + np.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    phi = 0.5 * _erfc(-g / math.sqrt(2))
    return g * phi, phi + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def distill(z, a, index, t, w):
    """(loss, gradient) of every row, float64."""
    z, a = np.asarray(z, np.float64), np.asarray(a, np.float64)
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    for r in range(rows):
        there = (index[r] >= 0) & (index[r] < vocab)
        if w[r] == 0 or not there.any():
            continue
        at = index[r][there]
        with np.errstate(all="ignore"):
            s = z[r] / t
            top = s.max()
            e = np.exp(s - top)
            log_q = s - top - np.log(e.sum())
            b = a[r][there] / t
            f = np.exp(b - b.max())
            p = f / f.sum()
            log_p = b - b.max() - np.log(f.sum())
            loss[r] = w[r] * t * t * np.where(p > 0, p * (log_p - log_q[at]), 0).sum()
            grad[r] = e / e.sum()
        np.subtract.at(grad[r], at, p)
        grad[r] *= w[r] * t
    return loss, grad

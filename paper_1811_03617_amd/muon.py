"""Newton-Schulz orthogonalisation and Muon's step (include/gvq.h, `gvq_orthogonalize`, `gvq_muon_step`).

    muon.step(weight, grad, buffer, lr=0.02)     # in place

Everything runs on the device's current stream; the workspace of a call comes from PyTorch's allocator on that stream.
"""
import numpy as np
import torch

from . import gvq
from .mx import _dtype, _matrix

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _coef(coefficients, steps):
    """(host array or None, number of steps) of a list of (a, b, c), one per step, or of the default polynomial."""
    if coefficients is None:
        return None, steps
    table = np.ascontiguousarray(coefficients, dtype=np.float64)
    if table.ndim != 2 or table.shape[1] != 3:
        raise ValueError("coefficients: triples (a, b, c), one for each step, are needed")
    return table, len(table)


def _workspace(batch, rows, cols, device):
    return torch.empty(gvq.gvq_orthogonalize_workspace(batch, rows, cols), dtype=torch.uint8, device=device)


def orthogonalize(g, steps=5, coefficients=None, eps=1e-7, dtype=None):
    """g ([rows, cols] or [batch, rows, cols]) with its singular values driven towards 1.  coefficients: (a, b, c) of every step
    instead of `steps` times the default."""
    if g.dim() not in (2, 3):
        raise ValueError(f"g: two or three dimensions are needed, not {g.dim()}")
    b = g if g.dim() == 3 else g.unsqueeze(0)
    batch, rows, cols = b.shape
    code, ld = _matrix(b[0], "g") if batch else (_dtype(g.dtype, "g"), cols)
    stride = b.stride(0) if batch > 1 else 0
    if stride < 0:
        raise ValueError("g: matrices have to lie one behind the other")
    out = torch.empty(g.shape, dtype=dtype or g.dtype, device=g.device)
    coef, steps = _coef(coefficients, steps)
    gvq.gvq_orthogonalize(g, code, batch, rows, cols, ld, stride, coef, steps, eps, out, _dtype(out.dtype, "dtype"), cols, rows * cols,
                          _workspace(batch, rows, cols, g.device))
    return out


def step(weight, grad, buffer, lr, momentum=0.95, weight_decay=0.0, nesterov=True, scale=None, steps=5, coefficients=None, eps=1e-7):
    """One step in place, of buffer (the momentum, float32) and weight (float32 or bfloat16): buffer <- momentum buffer + grad, and the
    weight moves against the orthogonalised buffer (nesterov: grad + momentum buffer).  scale: multiplies lr, sqrt(max(1, rows / cols))
    unless given."""
    code_w, ld_w = _matrix(weight, "weight")
    code_g, ld_g = _matrix(grad, "grad")
    code_m, ld_m = _matrix(buffer, "buffer")
    rows, cols = weight.shape
    if grad.shape != weight.shape or buffer.shape != weight.shape or code_m != gvq.F32:
        raise ValueError("grad and buffer: the weight's shape is needed, and float32 of the buffer")
    if scale is None:
        scale = max(1.0, rows / max(1, cols)) ** 0.5
    coef, steps = _coef(coefficients, steps)
    gvq.gvq_muon_step(weight, code_w, ld_w, grad, code_g, ld_g, buffer, ld_m, rows, cols, lr, momentum, weight_decay, int(nesterov), scale,
                      coef, steps, eps, _workspace(1, rows, cols, weight.device))

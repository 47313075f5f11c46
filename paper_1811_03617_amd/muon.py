"""Newton-Schulz orthogonalisation and Muon's step (include/gvq.h, `gvq_orthogonalize`, `gvq_muon_step`).

    muon.step(weight, grad, buffer, lr=0.02)     # in place

Everything runs on the device's current stream; the workspace of a call comes from PyTorch's allocator on that stream.  No gradient is
recorded: `orthogonalize` refuses a tensor that needs one, `step` is an optimiser's and takes weights that do.
"""
import numpy as np
import torch

from . import gvq
from .mx import _check, _dtype, _matrix, _no_graph, _now, _workspace

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _coef(coefficients, steps):
    """(host array or None, number of steps) of a list of (a, b, c), one per step, or of the default polynomial."""
    if coefficients is None:
        return None, steps
    table = np.ascontiguousarray(coefficients, dtype=np.float64)
    if table.ndim != 2 or table.shape[1] != 3:
        raise ValueError("coefficients: triples (a, b, c), one for each step, are needed")
    return table, len(table)


def orthogonalize(g, steps=5, coefficients=None, eps=1e-7, dtype=None):
    """g ([rows, cols] or [batch, rows, cols]) with its singular values driven towards 1.  coefficients: (a, b, c) of every step
    instead of `steps` times the default."""
    _no_graph(g, "g")
    if g.dim() not in (2, 3):
        raise ValueError(f"g: two or three dimensions are needed, not {g.dim()}")
    batch, rows, cols = g.shape if g.dim() == 3 else (1, *g.shape)
    code, ld, _, _ = _matrix(g if g.dim() == 2 else g[0], "g") if batch else (_dtype(g.dtype, "g"), cols, 0, 0)
    stride = g.stride(0) if batch > 1 else 0
    out = torch.empty(g.shape, dtype=dtype or g.dtype, device=g.device)
    coef, steps = _coef(coefficients, steps)
    ws = _workspace(g.device, "gvq_orthogonalize_workspace", batch, rows, cols)
    _check(gvq.lib().gvq_orthogonalize(g.data_ptr(), code, batch, rows, cols, ld, stride, coef if coef is None else coef.ctypes.data, steps,
                                       eps, out.data_ptr(), _dtype(out.dtype, "dtype"), cols, rows * cols, ws.data_ptr(), _now()),
           "gvq_orthogonalize")
    return out


def step(weight, grad, buffer, lr, momentum=0.95, weight_decay=0.0, nesterov=True, scale=None, steps=5, coefficients=None, eps=1e-7):
    """One step in place, of buffer (the momentum, float32) and weight (float32 or bfloat16): buffer <- momentum buffer + grad, and the
    weight moves against the orthogonalised buffer (nesterov: grad + momentum buffer).  scale: multiplies lr, sqrt(max(1, rows / cols))
    unless given."""
    code_w, ld_w, rows, cols = _matrix(weight, "weight")
    code_g, ld_g, rows_g, cols_g = _matrix(grad, "grad")
    code_b, ld_b, rows_b, cols_b = _matrix(buffer, "buffer")
    if (rows_g, cols_g) != (rows, cols) or (rows_b, cols_b) != (rows, cols) or code_b != gvq.F32:
        raise ValueError("grad and buffer: the weight's shape is needed, and float32 of the buffer")
    if scale is None:
        scale = max(1.0, rows / max(1, cols)) ** 0.5
    coef, steps = _coef(coefficients, steps)
    ws = _workspace(weight.device, "gvq_orthogonalize_workspace", 1, rows, cols)
    _check(gvq.lib().gvq_muon_step(weight.data_ptr(), code_w, ld_w, grad.data_ptr(), code_g, ld_g, buffer.data_ptr(), ld_b, rows, cols, lr,
                                   momentum, weight_decay, int(nesterov), scale, coef if coef is None else coef.ctypes.data, steps, eps,
                                   ws.data_ptr(), _now()), "gvq_muon_step")

"""4-bit microscaled matrices and the layers that keep their weights in them (include/gvq.h, `gvq_mx_*`).

    q, qt = mx.quantize_both(w)          # blocks along rows, and of the transpose
    y = mx.linear(x, q)                  # Q(x) W^T
    dx, dw = mx.linear_backward(dy, x, qt, noise=noise)

Tensors are two-dimensional, float32 or bfloat16, with neighbouring elements of a row next to each other; everything runs on the
device's current stream, and what a call allocates comes from PyTorch's allocator on that stream.
"""
from typing import NamedTuple

import torch

from . import gvq

_CODE = {torch.float32: gvq.F32, torch.bfloat16: gvq.BF16}


class MxMatrix(NamedTuple):
    """rows x cols numbers in blocks of 32 along a row: codes uint8 [rows][64 ceil(cols/128)], scales uint8 [rows][4 ceil(cols/128)]."""
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int


def _dtype(t, name):
    try:
        return _CODE[t]
    except KeyError:
        raise TypeError(f"{name}: float32 or bfloat16 is needed, not {t}") from None


def _matrix(t, name):
    """(dtype code, row stride) of a matrix on the current device."""
    if t.dim() != 2:
        raise ValueError(f"{name}: two dimensions are needed, not {t.dim()}")
    if t.device.type != "cuda" or t.device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: is not on the current GPU")
    code = _dtype(t.dtype, name)
    rows, cols = t.shape
    s0, s1 = t.stride()
    if (cols > 1 and s1 != 1) or (rows > 1 and s0 < cols):
        raise ValueError(f"{name}: neighbouring elements of a row have to be next to each other, and rows must not overlap")
    return code, (s0 if rows > 1 else cols)


def _bytes_of(t, name, rows, cols):
    """Row stride of random bytes for a rows x cols matrix."""
    if t.dtype != torch.uint8 or tuple(t.shape) != (rows, cols) or t.device.type != "cuda":
        raise ValueError(f"{name}: uint8 of shape ({rows}, {cols}) on the GPU is needed")
    s0, s1 = t.stride()
    if (cols > 1 and s1 != 1) or (rows > 1 and s0 < cols):
        raise ValueError(f"{name}: neighbouring elements of a row have to be next to each other")
    return s0 if rows > 1 else cols


def _stored(q, name, rows, cols):
    if (q.rows, q.cols) != (rows, cols):
        raise ValueError(f"{name}: {rows} x {cols} is needed, not {q.rows} x {q.cols}")
    k = -(-cols // 128)
    for t, n in ((q.codes, 64 * k), (q.scales, 4 * k)):
        if t.dtype != torch.uint8 or t.numel() != rows * n or not t.is_contiguous() or t.device.type != "cuda":
            raise ValueError(f"{name}: codes and scales are not those of a {rows} x {cols} matrix")


def _empty(rows, cols, device):
    k = -(-cols // 128)
    return MxMatrix(torch.empty(rows, 64 * k, dtype=torch.uint8, device=device),
                    torch.empty(rows, 4 * k, dtype=torch.uint8, device=device), rows, cols)


def _quantize(x, noise, along_rows, along_cols):
    code, ld = _matrix(x, "x")
    rows, cols = x.shape
    noise_ld = 0 if noise is None else _bytes_of(noise, "noise", rows, cols)
    q = _empty(rows, cols, x.device) if along_rows else None
    t = _empty(cols, rows, x.device) if along_cols else None
    gvq.gvq_mx_quantize(x, code, rows, cols, ld, noise, noise_ld, q and q.codes, q and q.scales, t and t.codes, t and t.scales)
    return q, t


def quantize(x, noise=None):
    """x in blocks along its rows, to the nearest; with `noise` (random uint8 of x's shape) stochastically."""
    return _quantize(x, noise, True, False)[0]


def quantize_columns(x, noise=None):
    """The transpose of x, in blocks along x's columns."""
    return _quantize(x, noise, False, True)[1]


def quantize_both(x, noise=None):
    """Both of these in one pass over x."""
    return _quantize(x, noise, True, True)


def dequantize(q, dtype=torch.float32):
    """The values that q stands for."""
    _stored(q, "q", q.rows, q.cols)
    out = torch.empty(q.rows, q.cols, dtype=dtype, device=q.codes.device)
    gvq.gvq_mx_dequantize(q.codes, q.scales, q.rows, q.cols, out, _dtype(dtype, "dtype"), q.cols)
    return out


def matmul(a, b, dtype=torch.float32, out=None, accumulate=False):
    """a b^T; with `out` into it, or added to it."""
    _stored(a, "a", a.rows, a.cols)
    _stored(b, "b", b.rows, a.cols)
    if out is None:
        if accumulate:
            raise ValueError("out: is needed to add to")
        out = torch.empty(a.rows, b.rows, dtype=dtype, device=a.codes.device)
    elif tuple(out.shape) != (a.rows, b.rows):
        raise ValueError(f"out: shape ({a.rows}, {b.rows}) is needed")
    code, ld = _matrix(out, "out")
    gvq.gvq_mx_matmul(a.codes, a.scales, b.codes, b.scales, a.rows, b.rows, a.cols, out, code, ld, int(accumulate))
    return out


def linear(x, w, dtype=None):
    """Q(x) W^T for a weight of n_out rows and n_in columns; the result's dtype is x's unless given."""
    code, ld = _matrix(x, "x")
    rows, n_in = x.shape
    _stored(w, "w", w.rows, n_in)
    y = torch.empty(rows, w.rows, dtype=dtype or x.dtype, device=x.device)
    ws = torch.empty(gvq.gvq_mx_linear_workspace(rows, n_in), dtype=torch.uint8, device=x.device)
    gvq.gvq_mx_linear(x, code, rows, n_in, ld, w.codes, w.scales, w.rows, y, _dtype(y.dtype, "dtype"), w.rows, ws)
    return y


def linear_backward(dy, x, wt, noise=None, dw=None, accumulate=False, dw_dtype=torch.float32, need_dx=True):
    """(dx, dw) of `linear`: wt is the weight's transpose in blocks along n_out.  dx has x's dtype (None unless needed), dw is given
    (and added to, if `accumulate`) or made."""
    code, ld_dy = _matrix(dy, "dy")
    code_x, ld_x = _matrix(x, "x")
    rows, n_out = dy.shape
    n_in = x.shape[1]
    if x.shape[0] != rows or code_x != code:
        raise ValueError("x: as many rows as dy, and its dtype, are needed")
    if need_dx:
        _stored(wt, "wt", n_in, n_out)
    noise_ld = 0 if noise is None else _bytes_of(noise, "noise", rows, n_out)
    dx = torch.empty(rows, n_in, dtype=x.dtype, device=x.device) if need_dx else None
    if dw is None:
        if accumulate:
            raise ValueError("dw: is needed to add to")
        dw = torch.empty(n_out, n_in, dtype=dw_dtype, device=x.device)
    elif tuple(dw.shape) != (n_out, n_in):
        raise ValueError(f"dw: shape ({n_out}, {n_in}) is needed")
    code_w, ld_dw = _matrix(dw, "dw")
    ws = torch.empty(gvq.gvq_mx_linear_backward_workspace(rows, n_in, n_out), dtype=torch.uint8, device=x.device)
    gvq.gvq_mx_linear_backward(dy, ld_dy, x, ld_x, code, rows, n_in, n_out, noise, noise_ld, wt.codes if need_dx else None,
                               wt.scales if need_dx else None, dx, code, n_in, dw, code_w, ld_dw, int(accumulate), ws)
    return dx, dw

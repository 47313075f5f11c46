"""Matrices in 8-bit integers with a scale for every row, the layers that keep their weights in them, and the gated block made of such
layers (include/gvq.h, `gvq_i8_*`).

    q, qt = i8.quantize_both(w)          # a scale for each row, and for each row of the transpose
    y = i8.linear(x, q)                  # Q(x) W^T, a scale for each token and each channel
    dx, dw = i8.linear_backward(dy, x, qt)
    h = i8.gated(x, q)                   # silu(g) u, [g | u] = Q(x) W^T
    dx, dw = i8.gated_backward(dh, x, q, qt)

Tensors are two-dimensional, float32 or bfloat16, with neighbouring elements of a row next to each other; everything runs on the
device's current stream, and what a call allocates comes from PyTorch's allocator on that stream.  No call records a gradient: one whose
result would need it is refused (wrap forward and backward in a torch.autograd.Function, where gradients are off; a Function's backward
under create_graph=True has them on).  Quantising a weight that needs one is not refused: what it gives carries none.
"""
import functools
from typing import NamedTuple

import torch

from . import gvq
from .mx import _check, _device, _dtype, _matrix, _no_graph, _now, _size

_ACTIVATIONS = {"silu": gvq.SILU, "gelu": gvq.GELU}


class I8Matrix(NamedTuple):
    """rows x cols numbers: codes int8 [rows][128 ceil(cols/128)], zeros behind the last column, and scales float32 [rows]."""
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int


def _stored(q, name, rows, cols):
    """(address of the codes, of the scales) of a rows x cols matrix in 8 bits."""
    codes, scales, r, c = q
    if r != rows or c != cols:
        raise ValueError(f"{name}: {rows} x {cols} is needed, not {r} x {c}")
    here = _device()   # (a tensor on the host says -1)
    if (codes.dtype is not torch.int8 or scales.dtype is not torch.float32 or codes.numel() != rows * (cols + 127 & -128) or scales.numel() != rows
            or not codes.is_contiguous() or not scales.is_contiguous() or codes.get_device() != here or scales.get_device() != here):
        raise ValueError(f"{name}: codes and scales are not those of a {rows} x {cols} matrix on the current GPU")
    _no_graph(scales, name)
    return codes.data_ptr(), scales.data_ptr()


def _empty(rows, cols, x):
    return I8Matrix(x.new_empty((rows, cols + 127 & -128), dtype=torch.int8), x.new_empty(rows, dtype=torch.float32), rows, cols)


def _space(x, name, *sizes):
    """A call's workspace.  (new_empty is a fifth faster than torch.empty with a dtype and a device, and small calls are as long as that.)"""
    return x.new_empty(_size(name, *sizes), dtype=torch.uint8)


def _written(t):
    """Autograd is told that a tensor of the caller's holds other numbers now: a backward pass that kept it will say so."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


def _activation(name):
    code = _ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation: one of {', '.join(_ACTIVATIONS)} is needed, not {name}")
    return code


def _quantize(x, along_rows, along_cols):
    code, ld, rows, cols = _matrix(x, "x")
    q = _empty(rows, cols, x) if along_rows else None
    t = _empty(cols, rows, x) if along_cols else None
    ws = _space(x, "gvq_i8_quantize_workspace", rows, cols) if along_cols else None
    _check(gvq.lib().gvq_i8_quantize(x.data_ptr(), code, rows, cols, ld, q and q[0].data_ptr(), q and q[1].data_ptr(), t and t[0].data_ptr(),
                                     t and t[1].data_ptr(), None if ws is None else ws.data_ptr(), _now()), "gvq_i8_quantize")
    return q, t


def quantize(x):
    """x with a scale for each of its rows."""
    return _quantize(x, True, False)[0]


def quantize_columns(x):
    """The transpose of x, with a scale for each of x's columns."""
    return _quantize(x, False, True)[1]


def quantize_both(x):
    """Both of these."""
    return _quantize(x, True, True)


def dequantize(q, dtype=torch.float32):
    """The values that q stands for."""
    rows, cols = q.rows, q.cols
    codes, scales = _stored(q, "q", rows, cols)
    out = torch.empty((rows, cols), dtype=dtype, device=q.codes.device)
    _check(gvq.lib().gvq_i8_dequantize(codes, scales, rows, cols, out.data_ptr(), _dtype(dtype, "dtype"), cols, _now()), "gvq_i8_dequantize")
    return out


def matmul(a, b, dtype=torch.float32, out=None, accumulate=False):
    """a b^T; with `out` into it, or added to it."""
    m, n, k = a.rows, b.rows, a.cols
    a_codes, a_scales = _stored(a, "a", m, k)
    b_codes, b_scales = _stored(b, "b", n, k)
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("out: is needed to add to")
        out = torch.empty((m, n), dtype=dtype, device=a.codes.device)
    _no_graph(out, "out")
    code, ld, rows, cols = _matrix(out, "out")
    if (rows, cols) != (m, n):
        raise ValueError(f"out: shape ({m}, {n}) is needed")
    _check(gvq.lib().gvq_i8_matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, out.data_ptr(), code, ld, int(accumulate), _now()),
           "gvq_i8_matmul")
    if given:
        _written(out)
    return out


def linear(x, w, dtype=None):
    """Q(x) W^T for a weight of n_out rows and n_in columns; the result's dtype is x's unless given."""
    _no_graph(x, "x")
    code, ld, rows, n_in = _matrix(x, "x")
    n_out = w.rows
    codes, scales = _stored(w, "w", n_out, n_in)
    y = x.new_empty((rows, n_out), dtype=dtype)
    ws = _space(x, "gvq_i8_linear_workspace", rows, n_in)
    _check(gvq.lib().gvq_i8_linear(x.data_ptr(), code, rows, n_in, ld, codes, scales, n_out, y.data_ptr(), _dtype(y.dtype, "dtype"), n_out,
                                   ws.data_ptr(), _now()), "gvq_i8_linear")
    return y


def _weight_gradient(dw, accumulate, dw_dtype, rows, cols, x, need_dx, need_dw):
    """(tensor, its address, dtype code, row stride) of dw, given or made; of none if it is not needed."""
    if not need_dw:
        if dw is not None or accumulate or not need_dx:
            raise ValueError("need_dw: has to be true where dw is given or added to, or dx is not needed either")
        return None, None, 0, cols
    if dw is None:
        if accumulate:
            raise ValueError("dw: is needed to add to")
        dw = x.new_empty((rows, cols), dtype=dw_dtype)
    _no_graph(dw, "dw")
    code, ld, r, c = _matrix(dw, "dw")
    if (r, c) != (rows, cols):
        raise ValueError(f"dw: shape ({rows}, {cols}) is needed")
    return dw, dw.data_ptr(), code, ld


@functools.lru_cache(maxsize=4096)
def _backward_bytes(rows, n_in, n_out, need_dx, need_dw):
    """Of a layer's workspace; what one gradient alone needs knows no limit for the other's sum."""
    if need_dx and need_dw:
        return _size("gvq_i8_linear_backward_workspace", rows, n_in, n_out)
    if need_dx:
        return _size("gvq_i8_linear_workspace", rows, n_out)
    return (_size("gvq_i8_linear_workspace", n_out, rows) + _size("gvq_i8_quantize_workspace", rows, n_out) +
            _size("gvq_i8_linear_workspace", n_in, rows) + _size("gvq_i8_quantize_workspace", rows, n_in))


def linear_backward(dy, x, wt, dw=None, accumulate=False, dw_dtype=torch.float32, need_dx=True, need_dw=True):
    """(dx, dw) of `linear`: wt is the weight's transpose with a scale for each of its rows.  dx has x's dtype (None unless needed), dw is
    given (and added to, if `accumulate`) or made (None unless needed).  dx sums n_out numbers and dw as many as there are rows: up to 131072,
    of the gradients that are needed."""
    _no_graph(dy, "dy")
    _no_graph(x, "x")
    code, ld_dy, rows, n_out = _matrix(dy, "dy")
    code_x, ld_x, rows_x, n_in = _matrix(x, "x")
    if rows_x != rows or code_x != code:
        raise ValueError("x: as many rows as dy, and its dtype, are needed")
    codes, scales = _stored(wt, "wt", n_in, n_out) if need_dx else (None, None)
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need_dx else None
    given = dw is not None
    dw, at_dw, code_w, ld_dw = _weight_gradient(dw, accumulate, dw_dtype, n_out, n_in, x, need_dx, need_dw)
    ws = x.new_empty(_backward_bytes(rows, n_in, n_out, need_dx, need_dw), dtype=torch.uint8)
    _check(gvq.lib().gvq_i8_linear_backward(dy.data_ptr(), ld_dy, x.data_ptr(), ld_x, code, rows, n_in, n_out, codes, scales,
                                            None if dx is None else dx.data_ptr(), code, n_in, at_dw, code_w, ld_dw,
                                            int(accumulate), ws.data_ptr(), _now()), "gvq_i8_linear_backward")
    if given:
        _written(dw)
    return dx, dw


def _halves(w):
    if w.rows % 2:
        raise ValueError(f"w: an even number of rows, the gate's and the other projection's, is needed, not {w.rows}")
    return w.rows // 2


def gated(x, w, activation="silu", dtype=None):
    """act(g) u with [g | u] = Q(x) W^T: the first half of w's rows is the gate's.  activation: "silu" or "gelu" (by the normal
    distribution itself); the result's dtype is x's unless given."""
    _no_graph(x, "x")
    act = _activation(activation)
    code, ld, rows, n_in = _matrix(x, "x")
    n = _halves(w)
    codes, scales = _stored(w, "w", 2 * n, n_in)
    h = x.new_empty((rows, n), dtype=dtype)
    ws = _space(x, "gvq_i8_linear_workspace", rows, n_in)
    _check(gvq.lib().gvq_i8_gated(x.data_ptr(), code, rows, n_in, ld, codes, scales, n, act, h.data_ptr(), _dtype(h.dtype, "dtype"), n,
                                  ws.data_ptr(), _now()), "gvq_i8_gated")
    return h


def _gated_inputs(dh, x, w):
    _no_graph(dh, "dh")
    _no_graph(x, "x")
    code, ld_dh, rows, n = _matrix(dh, "dh")
    code_x, ld_x, rows_x, n_in = _matrix(x, "x")
    if rows_x != rows or code_x != code:
        raise ValueError("x: as many rows as dh, and its dtype, are needed")
    codes, scales = _stored(w, "w", 2 * n, n_in)
    return code, ld_dh, ld_x, rows, n_in, n, codes, scales


def gated_gradient(dh, x, w, activation="silu"):
    """The gradient of [g | u] from that of `gated`'s result, in x's dtype: the dy of the layer that w is."""
    act = _activation(activation)
    code, ld_dh, ld_x, rows, n_in, n, codes, scales = _gated_inputs(dh, x, w)
    dg = x.new_empty((rows, 2 * n))
    ws = _space(x, "gvq_i8_linear_workspace", rows, n_in)
    _check(gvq.lib().gvq_i8_gated_gradient(dh.data_ptr(), ld_dh, x.data_ptr(), ld_x, code, rows, n_in, n, codes, scales, act, dg.data_ptr(),
                                           2 * n, ws.data_ptr(), _now()), "gvq_i8_gated_gradient")
    return dg


def gated_backward(dh, x, w, wt, activation="silu", dw=None, accumulate=False, dw_dtype=torch.float32, need_dx=True,
                   need_dw=True):
    """(dx, dw) of `gated`: linear_backward of gated_gradient.  wt is the transpose of all of w; dx, dw as there, dw of w's shape."""
    act = _activation(activation)
    code, ld_dh, ld_x, rows, n_in, n, codes, scales = _gated_inputs(dh, x, w)
    t_codes, t_scales = _stored(wt, "wt", n_in, 2 * n) if need_dx else (None, None)
    dx = torch.empty_like(x, memory_format=torch.contiguous_format) if need_dx else None
    given = dw is not None
    dw, at_dw, code_w, ld_dw = _weight_gradient(dw, accumulate, dw_dtype, 2 * n, n_in, x, need_dx, need_dw)
    size = (_size("gvq_i8_gated_backward_workspace", rows, n_in, n) if need_dx and need_dw else
            (8 * rows * n + 255 & -256) + max(_size("gvq_i8_linear_workspace", rows, n_in), _backward_bytes(rows, n_in, 2 * n, need_dx, need_dw)))
    ws = x.new_empty(size, dtype=torch.uint8)
    _check(gvq.lib().gvq_i8_gated_backward(dh.data_ptr(), ld_dh, x.data_ptr(), ld_x, code, rows, n_in, n, codes, scales, t_codes, t_scales, act,
                                           None if dx is None else dx.data_ptr(), code, n_in, at_dw, code_w, ld_dw, int(accumulate),
                                           ws.data_ptr(), _now()), "gvq_i8_gated_backward")
    if given:
        _written(dw)
    return dx, dw

"""4-bit microscaled matrices and the layers that keep their weights in them (include/gvq.h, `gvq_mx_*`).

    q, qt = mx.quantize_both(w)          # blocks along rows, and of the transpose
    y = mx.linear(x, q)                  # Q(x) W^T
    dx, dw = mx.linear_backward(dy, x, qt, noise=noise)

Tensors are two-dimensional, float32 or bfloat16, with neighbouring elements of a row next to each other; everything runs on the
device's current stream, and what a call allocates comes from PyTorch's allocator on that stream.  No call records a gradient: one whose
result would need it is refused (wrap linear and linear_backward in a torch.autograd.Function, where gradients are off).
"""
import functools
from typing import NamedTuple

import torch

from . import gvq

_CODE = {torch.float32: gvq.F32, torch.bfloat16: gvq.BF16}
_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream


class MxMatrix(NamedTuple):
    """rows x cols numbers in blocks of 32 along a row: codes uint8 [rows][64 ceil(cols/128)], scales uint8 [rows][4 ceil(cols/128)]."""
    codes: torch.Tensor
    scales: torch.Tensor
    rows: int
    cols: int


# Small calls are as long as what Python does around them: one look at each tensor, one call with plain numbers.

def _dtype(t, name):
    code = _CODE.get(t)
    if code is None:
        raise TypeError(f"{name}: float32 or bfloat16 is needed, not {t}")
    return code


def _matrix(t, name):
    """(dtype code, row stride, rows, columns) of a matrix on the current device."""
    if t.dim() != 2:
        raise ValueError(f"{name}: two dimensions are needed, not {t.dim()}")
    if not t.is_cuda or t.get_device() != _device():
        raise ValueError(f"{name}: is not on the current GPU")
    code = _dtype(t.dtype, name)
    rows, cols = t.shape
    s0, s1 = t.stride()
    if (cols > 1 and s1 != 1) or (rows > 1 and s0 < cols):
        raise ValueError(f"{name}: neighbouring elements of a row have to be next to each other, and rows must not overlap")
    return code, (s0 if rows > 1 else cols), rows, cols


def _no_graph(t, name):
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: needs a gradient, which this call does not record (detach it, or switch gradients off)")


def _noise(t, rows, cols):
    """(address, row stride) of random bytes for a rows x cols matrix, or of none."""
    if t is None:
        return None, 0
    if t.dtype != torch.uint8 or tuple(t.shape) != (rows, cols) or not t.is_cuda or t.get_device() != _device():
        raise ValueError(f"noise: uint8 of shape ({rows}, {cols}) on the current GPU is needed")
    s0, s1 = t.stride()
    if (cols > 1 and s1 != 1) or (rows > 1 and s0 < cols):
        raise ValueError("noise: neighbouring elements of a row have to be next to each other")
    return t.data_ptr(), (s0 if rows > 1 else cols)


def _stored(q, name, rows, cols):
    """(address of the codes, of the scales) of a rows x cols matrix in 4 bits."""
    codes, scales, r, c = q
    if r != rows or c != cols:
        raise ValueError(f"{name}: {rows} x {cols} is needed, not {r} x {c}")
    k = (cols + 127) // 128
    for t, n in ((codes, 64 * k), (scales, 4 * k)):
        if t.dtype != torch.uint8 or t.numel() != rows * n or not t.is_contiguous() or not t.is_cuda or t.get_device() != _device():
            raise ValueError(f"{name}: codes and scales are not those of a {rows} x {cols} matrix on the current GPU")
    return codes.data_ptr(), scales.data_ptr()


def _empty(rows, cols, device):
    k = (cols + 127) // 128
    return MxMatrix(torch.empty((rows, 64 * k), dtype=torch.uint8, device=device),
                    torch.empty((rows, 4 * k), dtype=torch.uint8, device=device), rows, cols)


def _now():
    return _raw_stream(_device())


def _check(status, where):
    if status != gvq.OK:
        raise gvq.GvqError(status, where)


@functools.lru_cache(maxsize=4096)
def _size(name, *sizes):
    """Bytes of a workspace."""
    return getattr(gvq, name)(*sizes)


def _workspace(device, name, *sizes):
    return torch.empty(_size(name, *sizes), dtype=torch.uint8, device=device)


def _quantize(x, noise, along_rows, along_cols):
    code, ld, rows, cols = _matrix(x, "x")
    z, z_ld = _noise(noise, rows, cols)
    q = _empty(rows, cols, x.device) if along_rows else None
    t = _empty(cols, rows, x.device) if along_cols else None
    _check(gvq.lib().gvq_mx_quantize(x.data_ptr(), code, rows, cols, ld, z, z_ld, q and q[0].data_ptr(), q and q[1].data_ptr(),
                                     t and t[0].data_ptr(), t and t[1].data_ptr(), _now()), "gvq_mx_quantize")
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
    rows, cols = q.rows, q.cols
    codes, scales = _stored(q, "q", rows, cols)
    out = torch.empty((rows, cols), dtype=dtype, device=q.codes.device)
    _check(gvq.lib().gvq_mx_dequantize(codes, scales, rows, cols, out.data_ptr(), _dtype(dtype, "dtype"), cols, _now()),
           "gvq_mx_dequantize")
    return out


def matmul(a, b, dtype=torch.float32, out=None, accumulate=False):
    """a b^T; with `out` into it, or added to it."""
    m, n, k = a.rows, b.rows, a.cols
    a_codes, a_scales = _stored(a, "a", m, k)
    b_codes, b_scales = _stored(b, "b", n, k)
    if out is None:
        if accumulate:
            raise ValueError("out: is needed to add to")
        out = torch.empty((m, n), dtype=dtype, device=a.codes.device)
    code, ld, rows, cols = _matrix(out, "out")
    if (rows, cols) != (m, n):
        raise ValueError(f"out: shape ({m}, {n}) is needed")
    _check(gvq.lib().gvq_mx_matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, out.data_ptr(), code, ld, int(accumulate), _now()),
           "gvq_mx_matmul")
    return out


def linear(x, w, dtype=None):
    """Q(x) W^T for a weight of n_out rows and n_in columns; the result's dtype is x's unless given."""
    _no_graph(x, "x")
    code, ld, rows, n_in = _matrix(x, "x")
    n_out = w.rows
    codes, scales = _stored(w, "w", n_out, n_in)
    y = torch.empty((rows, n_out), dtype=dtype or x.dtype, device=x.device)
    ws = _workspace(x.device, "gvq_mx_linear_workspace", rows, n_in)
    _check(gvq.lib().gvq_mx_linear(x.data_ptr(), code, rows, n_in, ld, codes, scales, n_out, y.data_ptr(), _dtype(y.dtype, "dtype"), n_out,
                                   ws.data_ptr(), _now()), "gvq_mx_linear")
    return y


def linear_backward(dy, x, wt, noise=None, dw=None, accumulate=False, dw_dtype=torch.float32, need_dx=True):
    """(dx, dw) of `linear`: wt is the weight's transpose in blocks along n_out.  dx has x's dtype (None unless needed), dw is given
    (and added to, if `accumulate`) or made."""
    code, ld_dy, rows, n_out = _matrix(dy, "dy")
    code_x, ld_x, rows_x, n_in = _matrix(x, "x")
    if rows_x != rows or code_x != code:
        raise ValueError("x: as many rows as dy, and its dtype, are needed")
    codes, scales = _stored(wt, "wt", n_in, n_out) if need_dx else (None, None)
    z, z_ld = _noise(noise, rows, n_out)
    dx = torch.empty((rows, n_in), dtype=x.dtype, device=x.device) if need_dx else None
    if dw is None:
        if accumulate:
            raise ValueError("dw: is needed to add to")
        dw = torch.empty((n_out, n_in), dtype=dw_dtype, device=x.device)
    code_w, ld_dw, rows_w, cols_w = _matrix(dw, "dw")
    if (rows_w, cols_w) != (n_out, n_in):
        raise ValueError(f"dw: shape ({n_out}, {n_in}) is needed")
    ws = _workspace(x.device, "gvq_mx_linear_backward_workspace", rows, n_in, n_out)
    _check(gvq.lib().gvq_mx_linear_backward(dy.data_ptr(), ld_dy, x.data_ptr(), ld_x, code, rows, n_in, n_out, z, z_ld, codes, scales,
                                            None if dx is None else dx.data_ptr(), code, n_in, dw.data_ptr(), code_w, ld_dw,
                                            int(accumulate), ws.data_ptr(), _now()), "gvq_mx_linear_backward")
    return dx, dw

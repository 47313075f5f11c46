"""The divergence of a teacher's top logits from a student's softmax, and its gradient (include/gvq.h, `gvq_distill`).

    losses, dlogits = distill.loss_and_gradient(logits, top, index, temperature=2.0, weight=weight)

For every row, with p = softmax(top / t) over the row's entries and q = softmax(logits / t) over all of the row:
loss = w t^2 sum_j p_j (log p_j - log q[index_j]), gradient = w t (q - p at its places); t is from 0.001 to 1000.  Everything runs on
the device's current stream.  No call records a gradient: `loss` refuses logits that need one, `loss_and_gradient` gives it; what the teacher's
logits or the weights would need is refused by both, and so is an `out` that needs one, unless it is the logits.
"""
import torch

from . import gvq
from .i8 import _written
from .mx import _check, _matrix, _device, _no_graph, _now, _size


def _run(logits, top, index, temperature, weight, grad, want):
    _no_graph(top, "top")
    if weight is not None:
        _no_graph(weight, "weight")
    code, ld, rows, vocab = _matrix(logits, "logits")
    code_top, ld_top, rows_top, n = _matrix(top, "top")
    if rows_top != rows or tuple(index.shape) != (rows, n) or index.dtype is not torch.int64 or index.get_device() != _device():
        raise ValueError("top and index: a row for each of logits' rows, of one length, and int64 of the index, are needed")
    s0, s1 = index.stride()
    if (n > 1 and s1 != 1) or (rows > 1 and s0 < n):
        raise ValueError("index: neighbouring elements of a row have to be next to each other, and rows must not overlap")
    if weight is not None and (weight.dtype is not torch.float32 or tuple(weight.shape) != (rows,) or not weight.is_contiguous()
                               or weight.get_device() != _device()):
        raise ValueError(f"weight: float32 of shape ({rows},), contiguous, on the current GPU is needed")
    ld_grad, given = vocab, grad is not None
    if want:
        if not given:
            grad = logits.new_empty((rows, vocab))
        else:
            if grad is not logits:
                _no_graph(grad, "out")
            code_g, ld_grad, rows_g, cols_g = _matrix(grad, "out")
            if (rows_g, cols_g) != (rows, vocab) or code_g != code:
                raise ValueError("out: the shape and dtype of logits are needed")
    losses = logits.new_empty(rows, dtype=torch.float32)
    size = _size("gvq_distill_workspace", rows, vocab, n)
    ws = logits.new_empty(size, dtype=torch.uint8) if size else None   # (most calls need none)
    _check(gvq.lib().gvq_distill(logits.data_ptr(), code, rows, vocab, ld, top.data_ptr(), code_top, index.data_ptr(), n, ld_top,
                                 s0 if rows > 1 else n, None if weight is None else weight.data_ptr(), temperature, losses.data_ptr(),
                                 grad.data_ptr() if want else None, ld_grad, None if ws is None else ws.data_ptr(), _now()), "gvq_distill")
    if given:
        _written(grad)
    return losses, grad


def loss(logits, top, index, temperature=1.0, weight=None):
    """Every row's loss, float32.  logits [rows, vocab], top [rows, n] the teacher's largest logits and index [rows, n] (int64) where they
    are; an index outside the vocabulary (-1, say) is no entry.  weight: float32 [rows], or 1; a row of weight 0 is not looked at."""
    _no_graph(logits, "logits")
    return _run(logits, top, index, temperature, weight, None, False)[0]


def loss_and_gradient(logits, top, index, temperature=1.0, weight=None, out=None):
    """(every row's loss, gradient of their sum by the logits in the logits' dtype).  out: where the gradient goes, the logits themselves
    if they are needed no more."""
    return _run(logits, top, index, temperature, weight, out, True)

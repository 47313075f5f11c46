"""Sizes and refusals of the 4-bit and Muon entry points that need no GPU: nothing here launches a kernel."""
import ctypes as C

import pytest

from paper_1811_03617_amd import gvq

A = 0x10000          # addresses that are only looked at
L = gvq.lib()


@pytest.mark.parametrize("rows,cols,codes,scales", [(0, 5, 0, 0), (3, 0, 0, 0), (1, 1, 64, 4), (7, 128, 448, 28), (7, 129, 896, 56),
                                                    (1 << 22, 1 << 22, 1 << 43, 1 << 39)])
def test_sizes_of_4_bit_matrices(rows, cols, codes, scales):
    assert gvq.gvq_mx_code_bytes(rows, cols) == codes
    assert gvq.gvq_mx_scale_bytes(rows, cols) == scales


def test_sizes_out_of_range():
    for f in (L.gvq_mx_code_bytes, L.gvq_mx_scale_bytes, L.gvq_mx_linear_workspace):
        assert f(-1, 5) == gvq.EINVAL and f(5, gvq.MX_MAX + 1) == gvq.EINVAL
    assert L.gvq_mx_linear_backward_workspace(5, 5, -2) == gvq.EINVAL
    assert L.gvq_orthogonalize_workspace(-1, 5, 5) == gvq.EINVAL
    assert L.gvq_orthogonalize_workspace(70000, 5, 5) == gvq.EINVAL
    assert L.gvq_orthogonalize_workspace(1, 40000, 40000) == gvq.EINVAL      # over 2^30 numbers
    with pytest.raises(gvq.GvqError):
        gvq.gvq_orthogonalize_workspace(1, 40000, 40000)


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 64, 64), (3, 64, 5000), (1, 65, 65), (5, 512, 4608), (1, 4096, 25088), (1, 25088, 4096)])
def test_workspaces_hold_what_a_matrix_needs(batch, rows, cols):
    n = gvq.gvq_orthogonalize_workspace(batch, rows, cols)
    assert n > 0
    if min(rows, cols) > 64:       # two planes of X, twice
        assert n >= batch * 8 * rows * cols
    assert gvq.gvq_orthogonalize_workspace(2 * batch, rows, cols) >= n


def test_4_bit_refusals():
    q = L.gvq_mx_quantize
    ok = [A, gvq.F32, 8, 64, 64, None, 0, A, A, None, None, None]

    def call(**change):
        args = list(ok)
        for k, v in change.items():
            args[int(k[1:])] = v
        return q(*args)
    for change in ({"_1": 2}, {"_2": -1}, {"_3": -1}, {"_4": 63}, {"_0": None}, {"_7": None}, {"_8": None}, {"_9": A}, {"_5": A, "_6": 63},
                   {"_3": gvq.MX_MAX + 1, "_4": gvq.MX_MAX + 1}):
        assert call(**change) == gvq.EINVAL, change
    for change in ({"_0": A + 2}, {"_7": A + 8}, {"_8": A + 1}, {"_9": A + 4, "_10": A}):
        assert call(**change) == gvq.EALIGN, change
    assert call(_2=0) == gvq.OK and call(_3=0, _4=0, _0=None) == gvq.OK
    assert L.gvq_mx_dequantize(A, A, 8, 64, A, gvq.F32, 63, None) == gvq.EINVAL
    assert L.gvq_mx_dequantize(A, A, 8, 64, A + 1, gvq.BF16, 64, None) == gvq.EALIGN
    assert L.gvq_mx_matmul(A, A, A, A, 8, 8, 64, None, gvq.F32, 8, 0, None) == gvq.EINVAL
    assert L.gvq_mx_matmul(A, A, A, A, 8, 8, 64, A, 9, 8, 0, None) == gvq.EINVAL
    assert L.gvq_mx_matmul(A, A + 4, A, A, 8, 8, 64, A, gvq.F32, 8, 0, None) == gvq.EALIGN
    assert L.gvq_mx_matmul(None, None, None, None, 0, 8, 64, None, gvq.F32, 8, 0, None) == gvq.OK
    assert L.gvq_mx_linear(A, gvq.F32, 8, 64, 60, A, A, 8, A, gvq.F32, 8, A, None) == gvq.EINVAL
    assert L.gvq_mx_linear(A, gvq.F32, 8, 64, 64, A, A, 8, A, gvq.F32, 7, A, None) == gvq.EINVAL
    assert L.gvq_mx_linear(A, gvq.F32, 8, 64, 64, A, A, 8, A, gvq.F32, 8, A + 2, None) == gvq.EALIGN
    assert L.gvq_mx_linear_backward(A, 7, A, 64, gvq.F32, 8, 64, 8, None, 0, A, A, A, gvq.F32, 64, A, gvq.F32, 64, 0, A, None) == gvq.EINVAL
    assert L.gvq_mx_linear_backward(A, 8, A, 64, gvq.F32, 8, 64, 8, A, 7, A, A, A, gvq.F32, 64, A, gvq.F32, 64, 0, A, None) == gvq.EINVAL
    assert L.gvq_mx_linear_backward(A, 8, None, 64, gvq.F32, 8, 64, 8, None, 0, A, A, A, gvq.F32, 64, A, gvq.F32, 64, 0, A, None) == gvq.EINVAL
    assert L.gvq_mx_linear_backward(A, 8, A, 64, gvq.F32, 8, 64, 8, None, 0, None, A, A, gvq.F32, 64, A, gvq.F32, 64, 0, A, None) == gvq.EINVAL


def test_muon_refusals():
    f = L.gvq_orthogonalize
    ok = [A, gvq.F32, 1, 80, 90, 90, 0, None, 5, 1e-7, A, gvq.F32, 90, 0, A, None]

    def call(**change):
        args = list(ok)
        for k, v in change.items():
            args[int(k[1:])] = v
        return f(*args)
    bad = (C.c_double * 3)(1.0, float("nan"), 0.0)
    for change in ({"_0": None}, {"_1": 4}, {"_2": -1}, {"_3": -1}, {"_5": 89}, {"_8": 0}, {"_8": 65}, {"_9": -1.0}, {"_9": float("inf")}, {"_10": None},
                   {"_11": 3}, {"_12": 89}, {"_14": None}, {"_2": 2, "_13": 100}, {"_6": -1}, {"_7": C.addressof(bad), "_8": 1}):
        assert call(**change) == gvq.EINVAL, change
    for change in ({"_0": A + 2}, {"_10": A + 1}, {"_14": A + 8}):
        assert call(**change) == gvq.EALIGN, change
    for change in ({"_2": 0}, {"_3": 0}, {"_4": 0}):
        assert call(**change) == gvq.OK, change
    g = L.gvq_muon_step
    ok2 = [A, gvq.F32, 90, A, gvq.F32, 90, A, 90, 80, 90, 0.1, 0.9, 0.0, 1, 1.0, None, 5, 1e-7, A, None]
    for k, v in ((0, None), (3, None), (6, None), (18, None), (1, 5), (4, 5), (2, 89), (5, 89), (7, 89), (10, float("inf")), (11, float("nan")),
                 (12, float("nan")), (14, float("inf")), (16, 0), (17, -1.0)):
        args = list(ok2)
        args[k] = v
        assert g(*args) == gvq.EINVAL, k
    for k, v in ((0, A + 2), (3, A + 1), (6, A + 2), (18, A + 4)):
        args = list(ok2)
        args[k] = v
        assert g(*args) == gvq.EALIGN, k


def test_a_gradient_that_is_not_wanted_asks_for_nothing():
    """What only dw needs (x, its type) is not looked at without dw, and what only dx needs (the weight) not without dx.  Sizes without elements: nothing runs."""
    f = L.gvq_mx_linear_backward
    odd, none = A + 1, 7          # an address of no type, a type that there is not
    assert f(A, 8, odd, 0, gvq.F32, 0, 64, 8, None, 0, A, A, A, gvq.F32, 64, None, none, 0, 0, A, None) == gvq.OK
    assert f(A, 0, A, 64, gvq.F32, 8, 64, 0, None, 0, odd, odd, None, none, 0, A, gvq.F32, 64, 0, A, None) == gvq.OK
    # and with them as before
    assert f(A, 8, odd, 64, gvq.F32, 0, 64, 8, None, 0, A, A, A, gvq.F32, 64, A, gvq.F32, 64, 0, A, None) == gvq.EALIGN
    assert f(A, 0, A, 64, gvq.F32, 8, 64, 0, None, 0, odd, A, A, gvq.F32, 64, A, gvq.F32, 64, 0, A, None) == gvq.EALIGN
    assert f(A, 8, A, 64, gvq.F32, 0, 64, 8, None, 0, A, A, A, gvq.F32, 64, A, none, 64, 0, A, None) == gvq.EINVAL
    assert f(A, 8, A, 64, gvq.F32, 0, 64, 8, None, 0, A, A, A, none, 64, None, gvq.F32, 64, 0, A, None) == gvq.EINVAL

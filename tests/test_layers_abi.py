"""Sizes and refusals of the 8-bit layers, the gated block and the loss that need no GPU: nothing here launches a kernel."""
import pytest

from paper_1811_03617_amd import gvq

A = 0x10000          # addresses that are only looked at
L = gvq.lib()
F, B = gvq.F32, gvq.BF16


def _caller(f, ok):
    def call(change):
        args = list(ok)
        for k, v in change.items():
            args[k] = v
        return f(*args)
    return call


def test_every_entry_point_is_there():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "gvq.h")).read()
    names = set(re.findall(r"\b(gvq_(?:i8|distill)\w*)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert len(names) == 15
    for n in names:
        assert hasattr(L, n) and hasattr(gvq, n), n


@pytest.mark.parametrize("rows,cols,codes", [(0, 5, 0), (3, 0, 0), (1, 1, 128), (7, 128, 896), (7, 129, 1792), (1 << 22, 1 << 22, 1 << 44)])
def test_sizes_of_8_bit_matrices(rows, cols, codes):
    assert gvq.gvq_i8_code_bytes(rows, cols) == codes


def test_sizes_out_of_range():
    for f in (L.gvq_i8_code_bytes, L.gvq_i8_quantize_workspace, L.gvq_i8_linear_workspace):
        assert f(-1, 5) == gvq.EINVAL and f(5, gvq.MX_MAX + 1) == gvq.EINVAL
    assert L.gvq_i8_linear_workspace(5, gvq.I8_MAX_SUM) > 0 and L.gvq_i8_linear_workspace(5, gvq.I8_MAX_SUM + 1) == gvq.EINVAL
    f = L.gvq_i8_linear_backward_workspace
    assert f(gvq.I8_MAX_SUM, 5, gvq.I8_MAX_SUM) > 0
    assert f(gvq.I8_MAX_SUM + 1, 5, 5) == gvq.EINVAL and f(5, 5, gvq.I8_MAX_SUM + 1) == gvq.EINVAL and f(5, -1, 5) == gvq.EINVAL
    g = L.gvq_i8_gated_backward_workspace
    assert g(5, 5, gvq.I8_MAX_SUM // 2) > 0 and g(5, 5, gvq.I8_MAX_SUM // 2 + 1) == gvq.EINVAL and g(5, gvq.I8_MAX_SUM + 1, 5) == gvq.EINVAL
    assert g(-1, 5, 5) == gvq.EINVAL and g(5, 5, -1) == gvq.EINVAL
    d = L.gvq_distill_workspace
    assert d(5, 5, -1) == gvq.EINVAL and d(5, 5, gvq.MAX_TOP + 1) == gvq.EINVAL and d(-1, 5, 5) == gvq.EINVAL and d(5, gvq.MX_MAX + 1, 5) == gvq.EINVAL
    with pytest.raises(gvq.GvqError):
        gvq.gvq_distill_workspace(5, 5, gvq.MAX_TOP + 1)


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 1, 1), (500, 4096, 1000), (4096, 25088, 4096), (131072, 64, 131072)])
def test_workspaces_hold_what_a_call_needs(rows, n_in, n_out):
    """Codes and scales of every operand that is quantised, and the maxima of the columns of two."""
    def codes(r, c):
        return r * ((c + 127) // 128 * 128) + 4 * r
    back = codes(rows, n_out) + codes(n_out, rows) + codes(n_in, rows)
    assert back + 4 * (n_in + n_out) <= gvq.gvq_i8_linear_backward_workspace(rows, n_in, n_out) <= back + 4 * 32 * (n_in + n_out) + 8 * 256
    if n_out <= gvq.I8_MAX_SUM // 2:
        both = gvq.gvq_i8_gated_backward_workspace(rows, n_in, n_out)
        assert both >= 8 * rows * n_out + gvq.gvq_i8_linear_backward_workspace(rows, n_in, 2 * n_out)


def test_the_loss_s_workspace_is_for_few_rows_of_many_logits():
    assert gvq.gvq_distill_workspace(4096, 131072, 64) == 0 and gvq.gvq_distill_workspace(16, 50021, 16) == 0 and gvq.gvq_distill_workspace(97, 131072, 16) == 0
    for rows, vocab in ((1, 65536), (1, 1 << 22), (16, 131072), (96, 262144)):
        n = gvq.gvq_distill_workspace(rows, vocab, 64)
        assert 0 < n <= 8 * rows * 256 + 256      # a thread of 256 joins each piece's two numbers


def test_quantiser_refusals():
    call = _caller(L.gvq_i8_quantize, [A, F, 8, 64, 64, A, A, None, None, None, None])
    for change in ({1: 2}, {2: -1}, {3: -1}, {4: 63}, {0: None}, {5: None}, {6: None}, {7: A}, {8: A}, {7: A, 8: A}, {3: gvq.MX_MAX + 1, 4: gvq.MX_MAX + 1}):
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 2}, {5: A + 8}, {6: A + 4}, {7: A + 4, 8: A, 9: A}, {7: A, 8: A + 4, 9: A}, {7: A, 8: A, 9: A + 8}):
        assert call(change) == gvq.EALIGN, change
    assert call({2: 0}) == gvq.OK and call({3: 0, 4: 0, 0: None}) == gvq.OK
    back = _caller(L.gvq_i8_dequantize, [A, A, 8, 64, A, F, 64, None])
    for change in ({0: None}, {1: None}, {4: None}, {2: -1}, {5: 7}, {6: 63}):
        assert back(change) == gvq.EINVAL, change
    for change in ({0: A + 8}, {1: A + 4}, {4: A + 2}):
        assert back(change) == gvq.EALIGN, change


def test_product_and_layer_refusals():
    call = _caller(L.gvq_i8_matmul, [A, A, A, A, 8, 8, 64, A, F, 8, 0, None])
    for change in ({0: None}, {1: None}, {2: None}, {3: None}, {7: None}, {8: 5}, {9: 7}, {4: -1}, {5: -1}, {6: -1}, {6: gvq.I8_MAX_SUM + 1}):
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 8}, {1: A + 4}, {2: A + 1}, {3: A + 8}, {7: A + 2}):
        assert call(change) == gvq.EALIGN, change
    assert call({4: 0}) == gvq.OK and call({5: 0, 9: 0}) == gvq.OK
    call = _caller(L.gvq_i8_linear, [A, F, 8, 64, 64, A, A, 8, A, B, 8, A, None])
    for change in ({0: None}, {5: None}, {6: None}, {8: None}, {11: None}, {1: 3}, {9: 3}, {4: 63}, {10: 7}, {2: -1}, {3: gvq.I8_MAX_SUM + 1, 4: gvq.MX_MAX},
                   {7: gvq.MX_MAX + 1, 10: gvq.MX_MAX + 1}):
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 2}, {5: A + 8}, {6: A + 4}, {8: A + 1}, {11: A + 8}):
        assert call(change) == gvq.EALIGN, change
    assert call({2: 0}) == gvq.OK and call({7: 0}) == gvq.OK


def test_backward_refusals():
    call = _caller(L.gvq_i8_linear_backward, [A, 8, A, 64, F, 8, 64, 8, A, A, A, F, 64, A, F, 64, 0, A, None])
    for change in ({0: None}, {1: 7}, {2: None}, {3: 63}, {4: 2}, {8: None}, {9: None}, {11: 2}, {12: 63}, {14: 2}, {15: 63}, {17: None}, {10: None, 13: None},
                   {5: gvq.I8_MAX_SUM + 1}, {7: gvq.I8_MAX_SUM + 1, 1: gvq.MX_MAX}):
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 2}, {2: A + 1}, {8: A + 8}, {9: A + 4}, {10: A + 2}, {13: A + 1}, {17: A + 8}):
        assert call(change) == gvq.EALIGN, change
    assert call({6: 0}) == gvq.OK
    # what only one gradient needs is not looked at when it is not wanted (sizes without elements: nothing runs)
    assert call({2: A + 1, 3: 0, 13: None, 14: 7, 15: 0, 5: 0}) == gvq.OK
    assert call({8: A + 1, 9: A + 1, 10: None, 11: 7, 12: 0, 7: 0, 1: 0}) == gvq.OK


def test_gated_refusals():
    call = _caller(L.gvq_i8_gated, [A, F, 8, 64, 64, A, A, 8, 0, A, F, 8, A, None])
    for change in ({8: 2}, {8: -1}, {0: None}, {5: None}, {6: None}, {9: None}, {12: None}, {4: 63}, {11: 7}, {7: gvq.MX_MAX // 2 + 1, 11: gvq.MX_MAX}):
        assert call(change) == gvq.EINVAL, change
    assert call({2: 0}) == gvq.OK
    call = _caller(L.gvq_i8_gated_gradient, [A, 8, A, 64, F, 8, 64, 8, A, A, 1, A, 16, A, None])
    for change in ({0: None}, {1: 7}, {2: None}, {3: 63}, {4: 9}, {8: None}, {9: None}, {10: 3}, {11: None}, {12: 15}, {13: None}):
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 2}, {2: A + 1}, {8: A + 8}, {9: A + 4}, {11: A + 2}, {13: A + 4}):
        assert call(change) == gvq.EALIGN, change
    # nothing is launched before everything has been looked at: these would run on addresses that are none
    call = _caller(L.gvq_i8_gated_backward, [A, 8, A, 64, F, 8, 64, 8, A, A, A, A, 1, A, F, 64, A, F, 64, 0, A, None])
    for change in ({0: None}, {1: 7}, {2: None}, {3: 63}, {4: 9}, {8: None}, {9: None}, {10: None}, {11: None}, {12: 3}, {14: 5}, {15: 63}, {17: 5}, {18: 63},
                   {20: None}, {13: None, 16: None}, {7: gvq.I8_MAX_SUM // 2 + 1, 1: gvq.MX_MAX}, {5: gvq.I8_MAX_SUM + 1}):
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 2}, {2: A + 1}, {8: A + 8}, {9: A + 4}, {10: A + 8}, {11: A + 8}, {13: A + 2}, {16: A + 2}, {20: A + 8}):
        assert call(change) == gvq.EALIGN, change
    assert call({6: 0}) == gvq.OK and call({5: 0, 7: 0}) == gvq.OK


def test_loss_refusals():
    call = _caller(L.gvq_distill, [A, F, 8, 100, 100, A, B, A, 5, 5, 5, A, 1.0, A, A, 100, None, None])
    for change in ({0: None}, {1: 4}, {2: -1}, {3: -1}, {4: 99}, {5: None}, {6: 3}, {7: None}, {8: -1}, {8: gvq.MAX_TOP + 1, 9: 2000, 10: 2000}, {9: 4}, {10: 4},
                   {15: 101}, {4: 101},                    # in place, with rows that start elsewhere
                   {12: 0.0}, {12: -1.0}, {12: float("nan")}, {12: float("inf")}, {12: 1e-4}, {12: 1e4}, {13: None}, {15: 99},
                   {3: 65536, 4: 65536, 15: 65536}):      # the last: few rows of many logits need a workspace
        assert call(change) == gvq.EINVAL, change
    for change in ({0: A + 2}, {5: A + 1}, {7: A + 4}, {11: A + 2}, {13: A + 2}, {14: A + 2}, {16: A + 8}):
        assert call(change) == gvq.EALIGN, change
    assert call({2: 0}) == gvq.OK

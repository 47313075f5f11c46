"""One gradient of an 8-bit layer without the other: only the axis that it sums has a limit.  Nothing here launches a kernel: there is a size of 0."""
import pytest

from paper_1811_03617_amd import gvq
from test_layers_abi import A, B, F, L, _caller

MORE = gvq.I8_MAX_SUM + 1
LAYER = _caller(L.gvq_i8_linear_backward, [A, gvq.MX_MAX, A, 64, F, 8, 0, 8, A, A, A, F, 64, A, F, 64, 0, A, None])
BLOCK = _caller(L.gvq_i8_gated_backward, [A, gvq.MX_MAX, A, 64, F, 8, 0, 8, A, A, A, A, 1, A, F, 64, A, F, 64, 0, A, None])


@pytest.mark.parametrize("call,dx,dw,n_out", [(LAYER, 10, 13, 7), (BLOCK, 13, 16, 7)])
def test_what_is_not_summed_has_no_limit(call, dx, dw, n_out):
    outputs = MORE if call is LAYER else MORE // 2 + 1
    assert call({5: MORE, dw: None}) == gvq.OK and call({n_out: outputs, dx: None}) == gvq.OK
    assert call({5: gvq.MX_MAX, dw: None}) == gvq.OK and call({n_out: gvq.MX_MAX // (1 if call is LAYER else 2), dx: None}) == gvq.OK
    for change in ({5: MORE}, {5: MORE, dx: None}, {n_out: outputs}, {n_out: outputs, dw: None}, {5: gvq.MX_MAX + 1, dw: None},
                   {n_out: gvq.MX_MAX + 1, dx: None}, {n_out: 1 << 62, dx: None}, {5: -1, dw: None}, {n_out: -1, dx: None}):
        assert call(change) == gvq.EINVAL, change


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 1, 1), (500, 4096, 1000), (131072, 64, 131072)])
def test_either_s_workspace_is_part_of_both_s(rows, n_in, n_out):
    one, peaks, both = gvq.gvq_i8_linear_workspace, gvq.gvq_i8_quantize_workspace, gvq.gvq_i8_linear_backward_workspace(rows, n_in, n_out)
    assert one(rows, n_out) + one(n_out, rows) + peaks(rows, n_out) + one(n_in, rows) + peaks(rows, n_in) == both

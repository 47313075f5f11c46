"""One gradient of an 8-bit layer or a gated block without the other: the same bits as with it, and past the limit of the other's sum."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
MOST = 131072


@pytest.fixture(scope="module")
def i8():
    from paper_1811_03617_amd import i8 as module
    return module


def _numbers(*shape, dtype=F32, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed + shape[0])).to(dtype).to(DEV)


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 5, 4), (33, 130, 70), (700, 300, 514), (1500, 64, 130)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_alone_and_together(i8, rows, n_in, n_out, dtype):
    x, dy, dh = _numbers(rows, n_in, dtype=dtype), _numbers(rows, n_out, dtype=dtype, seed=1), _numbers(rows, n_out // 2, dtype=dtype, seed=2)
    q, qt = i8.quantize_both(_numbers(n_out, n_in, seed=3))
    for both, dx, dw in ((i8.linear_backward(dy, x, qt), i8.linear_backward(dy, x, qt, need_dw=False), i8.linear_backward(dy, x, None, need_dx=False)),
                         (i8.gated_backward(dh, x, q, qt), i8.gated_backward(dh, x, q, qt, need_dw=False), i8.gated_backward(dh, x, q, None, need_dx=False))):
        assert dx[1] is None and dw[0] is None and torch.equal(dx[0], both[0]) and torch.equal(dw[1], both[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dx_of_more_tokens_than_dw_could_sum(i8, dtype):
    rows = MOST + 77
    x, dy, dh = _numbers(rows, 40, dtype=dtype), _numbers(rows, 130, dtype=dtype), _numbers(rows, 65, dtype=dtype)
    q, qt = i8.quantize_both(_numbers(130, 40))
    dx, none = i8.linear_backward(dy, x, qt, need_dw=False)
    assert none is None and torch.equal(dx[-200:], i8.linear_backward(dy[-200:], x[-200:], qt)[0])
    dx, none = i8.gated_backward(dh, x, q, qt, need_dw=False)
    assert none is None and torch.equal(dx[-200:], i8.gated_backward(dh[-200:], x[-200:], q, qt)[0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_dw_of_more_outputs_than_dx_could_sum(i8, dtype):
    """A head over a large vocabulary."""
    n = 151936
    x, dy = _numbers(30, 48, dtype=dtype), _numbers(30, n, dtype=dtype)
    none, dw = i8.linear_backward(dy, x, None, need_dx=False)
    assert none is None and torch.equal(dw[-200:], i8.linear_backward(dy[:, -200:], x, None, need_dx=False)[1])
    q = i8.quantize(_numbers(n, 48, seed=4))
    dh = dy[:, :n // 2].contiguous()
    none, dw = i8.gated_backward(dh, x, q, None, need_dx=False)
    dg = i8.gated_gradient(dh, x, q)
    assert none is None and torch.equal(dw, i8.linear_backward(dg, x, None, need_dx=False)[1])
    into = torch.ones_like(dw)
    i8.gated_backward(dh, x, q, None, need_dx=False, dw=into, accumulate=True)
    assert torch.equal(into, i8.linear_backward(dg, x, None, need_dx=False, dw=torch.ones_like(dw), accumulate=True)[1])


def test_refusals(i8):
    from paper_1811_03617_amd import gvq
    x, dy = _numbers(4, 10), _numbers(4, 6)
    q, qt = i8.quantize_both(_numbers(6, 10))
    dw = torch.zeros(6, 10, device=DEV)
    for more in (dict(dw=dw), dict(accumulate=True), dict(need_dx=False)):
        with pytest.raises(ValueError):
            i8.linear_backward(dy, x, qt, need_dw=False, **more)
        with pytest.raises(ValueError):
            i8.gated_backward(dy[:, :3].contiguous(), x, q, qt, need_dw=False, **more)
    far = torch.zeros(MOST + 1, 6, device=DEV)
    for more in (dict(), dict(need_dx=False)):
        with pytest.raises(gvq.GvqError):
            i8.linear_backward(far, torch.zeros(MOST + 1, 10, device=DEV), qt, **more)

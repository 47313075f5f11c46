"""Matrices whose places pass 2^31 elements and 2^32 bytes: their last rows and columns against the same ones alone, bit for bit (whole numbers
are added, so that a row's result does not depend on how many there are)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def i8():
    from paper_1811_03617_amd import i8 as module
    return module


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def _numbers(rows, cols, dtype=BF16):
    torch.manual_seed(rows + cols)
    return torch.empty((rows, cols), dtype=dtype, device=DEV).normal_()


def _same(q, r):
    return torch.equal(q.codes, r.codes) and torch.equal(q.scales, r.scales)


def test_quantising_both_ways(i8):
    rows, cols = 140001, 32768               # 4.6e9 numbers
    x = _numbers(rows, cols)
    q, t = i8.quantize_both(x)
    last = i8.quantize(x[-70:])
    assert torch.equal(q.codes[-70:], last.codes) and torch.equal(q.scales[-70:], last.scales)
    edge = i8.quantize_columns(x[:, -40:])
    assert torch.equal(t.codes[-40:], edge.codes) and torch.equal(t.scales[-40:], edge.scales)
    back = i8.dequantize(q, BF16)
    assert torch.equal(back[-70:], i8.dequantize(last, BF16))


def test_layers_of_many_rows(i8):
    rows, n_in = 1100003, 4096               # 4.5e9 numbers and codes
    x = _numbers(rows, n_in)
    q, qt = i8.quantize_both(_numbers(34, n_in, F32))
    y = i8.linear(x, q)
    assert torch.equal(y[-300:], i8.linear(x[-300:].clone(), q))
    h = i8.gated(x, q)
    assert torch.equal(h[-300:], i8.gated(x[-300:].clone(), q))


def test_results_of_many_numbers(i8):
    rows, n_out = 70001, 65536               # 4.6e9 results
    x, w = _numbers(rows, 64), _numbers(n_out, 64, F32)
    q = i8.quantize(w)
    y = i8.linear(x, q)
    assert torch.equal(y[-130:], i8.linear(x[-130:].clone(), q))
    del y
    h = i8.gated(x, q)
    dg = i8.gated_gradient(h, x, q)
    some = x[-130:].clone()
    assert torch.equal(h[-130:], i8.gated(some, q)) and torch.equal(dg[-130:], i8.gated_gradient(h[-130:].clone(), some, q))


def test_gradients_of_many_numbers(i8):
    rows, n_in, n_out = 20, 65540, 70001     # dw: 4.6e9 numbers
    x, dy = _numbers(rows, n_in), _numbers(rows, n_out)
    _, dw = i8.linear_backward(dy, x, None, dw_dtype=BF16, need_dx=False)
    _, some = i8.linear_backward(dy[:, -90:].clone(), x, None, dw_dtype=BF16, need_dx=False)
    assert torch.equal(dw[-90:], some)
    i8.linear_backward(dy, x, None, dw=dw, accumulate=True, need_dx=False)
    i8.linear_backward(dy[:, -90:].clone(), x, None, dw=some, accumulate=True, need_dx=False)
    assert torch.equal(dw[-90:], some)


@pytest.mark.parametrize("rows,vocab", [(33001, 131072), (1100008, 4001)])
def test_losses_of_many_logits(rows, vocab):
    from paper_1811_03617_amd import distill
    z = _numbers(rows, vocab)                # 4.3e9 logits
    top = _numbers(rows, 8, F32)
    index = torch.randint(0, vocab, (rows, 8), device=DEV)
    some = z[-200:].clone()
    want = distill.loss_and_gradient(some, top[-200:], index[-200:], temperature=2.0)
    losses, grad = distill.loss_and_gradient(z, top, index, temperature=2.0, out=z)
    assert torch.equal(losses[-200:], want[0])
    assert torch.equal(grad[-200:], want[1])

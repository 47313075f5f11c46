"""What the 8-bit layers, the gated block and the loss do about gradients that they do not record."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _numbers(*shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(shape[0])).to(DEV)


def _case():
    from paper_1811_03617_amd import i8
    x, dy, dh = _numbers(4, 10), _numbers(4, 6), _numbers(4, 3)
    return (i8, x, dy, dh, *i8.quantize_both(_numbers(6, 10)))


def _asks(t):
    return t.clone().requires_grad_()


def _scales(q):
    return q._replace(scales=_asks(q.scales))


CALLS = {
    "linear_backward, dy": lambda i8, x, dy, dh, q, qt: i8.linear_backward(_asks(dy), x, qt),
    "linear_backward, x": lambda i8, x, dy, dh, q, qt: i8.linear_backward(dy, _asks(x), qt),
    "linear_backward, dw": lambda i8, x, dy, dh, q, qt: i8.linear_backward(dy, x, qt, dw=_asks(_numbers(6, 10))),
    "gated_gradient, dh": lambda i8, x, dy, dh, q, qt: i8.gated_gradient(_asks(dh), x, q),
    "gated_gradient, x": lambda i8, x, dy, dh, q, qt: i8.gated_gradient(dh, _asks(x), q),
    "gated_backward, dh": lambda i8, x, dy, dh, q, qt: i8.gated_backward(_asks(dh), x, q, qt),
    "gated_backward, x": lambda i8, x, dy, dh, q, qt: i8.gated_backward(dh, _asks(x), q, qt),
    "gated_backward, dw": lambda i8, x, dy, dh, q, qt: i8.gated_backward(dh, x, q, qt, dw=_asks(_numbers(6, 10)), accumulate=True),
    "matmul, out": lambda i8, x, dy, dh, q, qt: i8.matmul(q, q, out=_asks(_numbers(6, 6))),
    "matmul, scales": lambda i8, x, dy, dh, q, qt: i8.matmul(q, _scales(q)),
    "linear, scales": lambda i8, x, dy, dh, q, qt: i8.linear(x, _scales(q)),
    "linear_backward, scales": lambda i8, x, dy, dh, q, qt: i8.linear_backward(dy, x, _scales(qt)),
    "gated, scales": lambda i8, x, dy, dh, q, qt: i8.gated(x, _scales(q)),
    "dequantize, scales": lambda i8, x, dy, dh, q, qt: i8.dequantize(_scales(q)),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_a_result_that_would_need_a_gradient_is_refused(name):
    case = _case()
    with pytest.raises(ValueError):
        CALLS[name](*case)
    with torch.no_grad():
        CALLS[name](*case)


def test_an_out_of_the_loss_that_needs_one_is_refused_unless_it_is_the_logits():
    from paper_1811_03617_amd import distill
    z, top, index = _numbers(4, 50), _numbers(4, 3), torch.zeros(4, 3, dtype=torch.int64, device=DEV)
    with pytest.raises(ValueError):
        distill.loss_and_gradient(z, top, index, out=_asks(z))
    want = distill.loss_and_gradient(z, top, index)
    leaf = _numbers(50, 50).requires_grad_()
    logits = z @ leaf
    got = distill.loss_and_gradient(logits, top, index, out=logits)
    assert got[1] is logits
    logits.backward(got[1].detach())           # the product does not look at its result
    assert torch.isfinite(leaf.grad).all() and want[0].shape == got[0].shape


def test_a_second_derivative_is_refused_and_the_first_is_not():
    i8, x, dy, dh, _, _ = _case()

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            q, ctx.qt = i8.quantize_both(weight)
            ctx.save_for_backward(x)
            return i8.linear(x, q)

        @staticmethod
        def backward(ctx, dy):
            return i8.linear_backward(dy, ctx.saved_tensors[0], ctx.qt)

    x, w = x.requires_grad_(), _numbers(6, 10).requires_grad_()
    y = Layer.apply(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    with pytest.raises(ValueError):
        torch.autograd.grad(y, (x, w), dy, create_graph=True)
    i8.quantize_both(w)                        # a weight itself is quantised with gradients on


def test_what_autograd_kept_is_not_written_unseen():
    """A tensor that is written into is another one for a backward pass that needs its numbers."""
    from paper_1811_03617_amd import distill
    i8, x, dy, dh, q, qt = _case()
    z, top, index = _numbers(6, 10), _numbers(6, 3), torch.zeros(6, 3, dtype=torch.int64, device=DEV)
    writes = {
        "matmul": ((6, 6), lambda t: i8.matmul(q, q, out=t)),
        "linear_backward": ((6, 10), lambda t: i8.linear_backward(dy, x, qt, dw=t, accumulate=True)),
        "gated_backward": ((6, 10), lambda t: i8.gated_backward(dh, x, q, None, dw=t, need_dx=False)),
        "loss_and_gradient": ((6, 10), lambda t: distill.loss_and_gradient(z, top, index, out=t)),
    }
    for name, (shape, write) in writes.items():
        kept, leaf = _numbers(*shape), torch.ones(shape, device=DEV, requires_grad=True)
        y = (leaf * kept).sum()
        before = kept._version
        write(kept)
        assert kept._version > before, name
        with pytest.raises(RuntimeError):
            y.backward()
    leaf = torch.ones(10, 10, device=DEV, requires_grad=True)
    logits = z @ leaf
    y = logits.square().sum()
    distill.loss_and_gradient(logits, top, index, out=logits)
    with pytest.raises(RuntimeError):
        y.backward()
    with torch.inference_mode():               # tensors that count no versions
        for name, (shape, write) in writes.items():
            write(torch.zeros(shape, device=DEV))

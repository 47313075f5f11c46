"""4-bit layers and Muon inside a program that uses automatic gradients."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def calls():
    from paper_1811_03617_amd import muon, mx
    return mx, muon


def test_what_would_lose_a_gradient_is_refused(calls):
    mx, muon = calls
    x = torch.randn(5, 64, device=DEV, requires_grad=True)
    q = mx.quantize(torch.randn(8, 64, device=DEV))
    with pytest.raises(ValueError, match="gradient"):
        mx.linear(x, q)
    with pytest.raises(ValueError, match="gradient"):
        muon.orthogonalize(x)
    want = mx.linear(x.detach(), q)
    with torch.no_grad():
        assert torch.equal(mx.linear(x, q), want)
        muon.orthogonalize(x)


def test_a_layer_in_an_autograd_function(calls):
    """As the refusal says: forward and backward in a Function, weights that need a gradient in quantize and in Muon's step."""
    mx, muon = calls

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            q, ctx.qt = mx.quantize_both(weight)
            ctx.save_for_backward(x)
            return mx.linear(x, q)

        @staticmethod
        def backward(ctx, dy):
            return mx.linear_backward(dy.contiguous(), ctx.saved_tensors[0], ctx.qt)

    x = torch.randn(33, 64, device=DEV, requires_grad=True)
    w = torch.nn.Parameter(torch.randn(40, 64, device=DEV))
    c = torch.randn(33, 40, device=DEV)
    (Layer.apply(x, w) * c).sum().backward()
    dx, dw = mx.linear_backward(c, x.detach(), mx.quantize_columns(w.detach()))
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw)
    buffer = torch.zeros_like(w.grad)
    before = w.detach().clone()
    muon.step(w, w.grad, buffer, lr=0.1)
    assert torch.equal(buffer, w.grad) and not torch.equal(w.detach(), before)

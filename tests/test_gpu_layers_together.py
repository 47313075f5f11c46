"""The 8-bit layers, the gated block, the loss and Muon's step in one program, as examples/distill_8bit.py has them: each stage against its
definition on what the stage before it gave, the whole gradient against a float64 network's and against differences of its loss."""
import importlib.util
import os

import numpy as np
import pytest

import _layers_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_8bit", os.path.join(ROOT, "examples", "distill_8bit.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _np(x):
    return x.detach().float().cpu().numpy()


def _case(example, rows, dtype, seed=3):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    teacher, student = example.network(gen), example.network(gen)
    x = torch.randn(rows, example.WIDTH, generator=gen, device=DEV).to(dtype)
    top, index = example.tell(teacher, x)
    return student, x, top, index, torch.full((rows,), 1.0 / rows, device=DEV)


@pytest.mark.parametrize("rows", [3, 61])
def test_each_stage_on_what_the_one_before_gave(example, rows):
    from paper_1811_03617_amd import distill, i8
    (both, down, head), x, top, index, weight = _case(example, rows, torch.float32)
    h = i8.gated(x, both.q)
    s = ref.product(ref.integers(_np(x)), ref.integers(_np(both.weight))).astype(np.float64)
    g, u = s[:, :example.HIDDEN], s[:, example.HIDDEN:]
    value, slope = ref.activation(g, "silu")
    assert (np.abs(_np(h) - value * u) <= np.abs(value * u) * ref.F32_HALF * (60 + 8 * np.abs(g))).all()
    y, z = i8.linear(h, down.q), None
    assert np.array_equal(_np(y), ref.product(ref.integers(_np(h)), ref.integers(_np(down.weight))))
    z = i8.linear(y, head.q)
    assert np.array_equal(_np(z), ref.product(ref.integers(_np(y)), ref.integers(_np(head.weight))))
    losses, dz = distill.loss_and_gradient(z, top, index, temperature=example.TEMPERATURE, weight=weight)
    want = ref.distill(_np(z), _np(top), index.cpu().numpy(), example.TEMPERATURE, _np(weight).astype(np.float64))
    assert np.allclose(_np(losses), want[0], rtol=1e-5) and np.allclose(_np(dz), want[1], rtol=1e-4, atol=1e-6 * np.abs(want[1]).max())
    dy, d_head = i8.linear_backward(dz, y, head.qt)
    assert np.array_equal(_np(dy), ref.product(ref.integers(_np(dz)), ref.integers(_np(head.weight).T)))
    assert np.array_equal(_np(d_head), ref.product(ref.integers(_np(dz).T), ref.integers(_np(y).T)))
    dh, d_down = i8.linear_backward(dy, h, down.qt)
    dg = i8.gated_gradient(dh, x, both.q)
    _, d_both = i8.gated_backward(dh, x, both.q, None, need_dx=False)
    assert np.array_equal(_np(d_both), ref.product(ref.integers(_np(dg).T), ref.integers(_np(x).T)))
    got = example.gradients([both, down, head], x, top, index, weight)
    for a, b in zip(got[1], (d_both, d_down, d_head)):
        assert torch.equal(a, b)
    assert torch.equal(got[0], losses)


def _float64(example, weights, x, top, index, weight):
    """The sum of the losses of the same network in float64, nothing quantised."""
    both, down, head = weights
    g, u = (x.double() @ both.t()).chunk(2, 1)
    z = ((torch.nn.functional.silu(g) * u) @ down.t()) @ head.t()
    t = example.TEMPERATURE
    p = torch.softmax(top.double() / t, 1)
    return (weight.double() * t * t * (p * (torch.log(p) - torch.log_softmax(z / t, 1).gather(1, index))).sum(1)).sum()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_whole_gradient(example, dtype):
    """Each quantised operand is off by half a step at most, uniformly: its largest number / 127 / sqrt(12) rms, for normal numbers whose largest of
    some hundred are 3 to 4 times their rms 0.9 % of it.  A product's two operands are off independently, 1.3 %; the logits' path has three
    products and the gradient's path three more, and the softmax's sensitivity is of the order of 1 (logits of the order of 1, t = 2): 3 to 4 %
    altogether, more for output gradients whose largest number stands out, 10 times their rms, 2.3 %.  A tenth is asked for."""
    student, x, top, index, weight = _case(example, 384, dtype)
    losses, grads = example.gradients(student, x, top, index, weight)
    weights = [layer.weight.double().requires_grad_() for layer in student]
    loss = _float64(example, weights, x, top, index, weight)
    want = torch.autograd.grad(loss, weights)
    assert abs(losses.double().sum() - loss) <= 0.05 * loss
    for got, w in zip(grads, want):
        assert torch.linalg.vector_norm(got.double() - w) <= 0.1 * torch.linalg.vector_norm(w)
    # and along the 8-bit gradient the float64 loss falls as fast as that gradient says
    with torch.no_grad():
        step = 1e-3 / float(sum(g.double().square().sum() for g in grads)) ** 0.5
        up, down = (_float64(example, [w + s * step * g.double() for w, g in zip(weights, grads)], x, top, index, weight) for s in (1, -1))
        rate = float(up - down) / (2 * step)
        assert abs(rate - float(sum(g.double().square().sum() for g in grads))) <= 0.1 * rate


def test_training_runs_and_repeats_bit_for_bit(example):
    a = example.train(steps=8, tell_loss=lambda *_: None)
    b = example.train(steps=8, tell_loss=lambda *_: None)
    assert a == b and all(l == l and l < float("inf") for l in a)


def test_a_step_in_an_autograd_function(example):
    """As the refusals say: forward and backward in Functions, where gradients are off."""
    from paper_1811_03617_amd import distill, i8

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            q, ctx.qt = i8.quantize_both(weight)
            ctx.save_for_backward(x)
            return i8.linear(x, q)

        @staticmethod
        def backward(ctx, dy):
            return i8.linear_backward(dy.contiguous(), ctx.saved_tensors[0], ctx.qt)

    class Gated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            ctx.q, ctx.qt = i8.quantize_both(weight)
            ctx.save_for_backward(x)
            return i8.gated(x, ctx.q)

        @staticmethod
        def backward(ctx, dh):
            return i8.gated_backward(dh.contiguous(), ctx.saved_tensors[0], ctx.q, ctx.qt)

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, z, top, index, weight):
            losses, grad = distill.loss_and_gradient(z, top, index, temperature=2.0, weight=weight)
            ctx.save_for_backward(grad)
            return losses.sum()

        @staticmethod
        def backward(ctx, d):
            return d * ctx.saved_tensors[0], None, None, None

    (both, down, head), x, top, index, weight = _case(example, 40, torch.float32)
    leaves = [layer.weight.clone().requires_grad_() for layer in (both, down, head)]
    Loss.apply(Layer.apply(Layer.apply(Gated.apply(x, leaves[0]), leaves[1]), leaves[2]), top, index, weight).backward()
    _, grads = example.gradients([both, down, head], x, top, index, weight)
    assert all(torch.equal(leaf.grad, g) for leaf, g in zip(leaves, grads))


def test_two_streams_at_one_time():
    """Calls that run side by side share nothing: each has its own workspace, from its own stream."""
    from paper_1811_03617_amd import distill, i8
    gen = torch.Generator(device=DEV).manual_seed(9)

    def numbers(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)
    sets = []
    for rows in (500, 1300):
        _, wt = i8.quantize_both(numbers(600, 700))
        gate, gate_t = i8.quantize_both(numbers(900, 700))
        logits, top = numbers(9, 70001), numbers(9, 5)
        index = torch.randint(0, 70001, (9, 5), generator=gen, device=DEV)
        sets.append((numbers(rows, 700), numbers(rows, 600), numbers(rows, 450), wt, gate, gate_t, logits, top, index))

    def pass_(x, dy, dh, wt, gate, gate_t, logits, top, index):
        return (*i8.linear_backward(dy, x, wt), i8.gated(x[:3], gate), *i8.gated_backward(dh, x, gate, gate_t), *distill.loss_and_gradient(logits, top, index))
    want = [pass_(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for stream in streams:
        stream.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[k].append(pass_(*sets[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for one in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(one, want[k]))

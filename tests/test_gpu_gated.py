"""The gated block: against its definition in float64, its gradients against the formula's and against differences."""
import numpy as np
import pytest

import _layers_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def i8():
    from paper_1811_03617_amd import i8 as module
    return module


def _np(x):
    return x.detach().float().cpu().numpy()


def _case(rows, n_in, n, dtype, spread=1.0, seed=0):
    gen = torch.Generator().manual_seed(seed + rows)
    x = (torch.randn(rows, n_in, generator=gen) * torch.exp(0.5 * torch.randn(rows, 1, generator=gen))).to(dtype)
    w = spread * torch.randn(2 * n, n_in, generator=gen) / n_in ** 0.5
    dh = (torch.randn(rows, n, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen))).to(dtype)
    return x, w, dh


def _sums(x, w):
    """g and u as float32 numbers, which the kernel's are to the bit."""
    s = ref.product(ref.integers(_np(x)), ref.integers(_np(w)))
    n = s.shape[1] // 2
    return s[:, :n].astype(np.float64), s[:, n:].astype(np.float64)


# What the activation's own arithmetic may be off, relative, in halves of float32 steps: the exponential (its argument is rounded, which counts
# |g| times, and |g| up to 20 matters before the result is negligible: 30 + 2), a division or erfc (16 by its documented bound), products.
def _room(g):
    return ref.F32_HALF * (60 + 4 * np.minimum(np.abs(g), 90) * np.maximum(1, np.minimum(np.abs(g), 14) / 2))


SIZES = [(1, 1, 1), (1, 300, 100), (2, 128, 17), (4, 1000, 130), (5, 64, 64), (17, 260, 33), (100, 129, 70), (300, 500, 257)]


@pytest.mark.parametrize("rows,n_in,n", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_forward(i8, rows, n_in, n, dtype, act):
    x, w, _ = _case(rows, n_in, n, dtype, 3.0)
    g, u = _sums(x, w)
    q = i8.quantize(w.to(DEV))
    want = ref.activation(g, act)[0] * u
    for out in (F32, BF16):
        got = _np(i8.gated(x.to(DEV), q, activation=act, dtype=out))
        room = np.abs(want) * (_room(g) + (ref.BF16_HALF if out == BF16 else 0)) + 1e-30
        assert (np.abs(got - want) <= room).all()
    assert i8.gated(x.to(DEV), q, activation=act).dtype == dtype


@pytest.mark.parametrize("rows,n_in,n", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_of_the_sums(i8, rows, n_in, n, dtype, act):
    x, w, dh = _case(rows, n_in, n, dtype, 3.0)
    g, u = _sums(x, w)
    got = _np(i8.gated_gradient(dh.to(DEV), x.to(DEV), i8.quantize(w.to(DEV)), activation=act))
    value, slope = ref.activation(g, act)
    d = _np(dh).astype(np.float64)
    last = ref.BF16_HALF if dtype == BF16 else 0
    # the slope is a sum of two terms that may cancel: their sizes count, not the sum's
    size = 1 / (1 + np.exp(-g)) * (1 + np.abs(g)) if act == "silu" else np.abs(slope) + np.abs(g) * np.exp(-g * g / 2)
    want = d * u * slope
    assert (np.abs(got[:, :n] - want) <= np.abs(want) * last + np.abs(d * u) * size * _room(g) * (1 + last) + 1e-30).all()
    want = d * value
    assert (np.abs(got[:, n:] - want) <= np.abs(want) * (_room(g) + last) * (1 + last) + 1e-30).all()
    # and the formula's slope is that of the formula's value
    step = 1e-5
    near = (ref.activation(g + step, act)[0] - ref.activation(g - step, act)[0]) / (2 * step)
    assert (np.abs(near - slope) <= 1e-8).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_sums_from_nothing_to_far_out(i8, act):
    """Gates of -200 to 200, at which the exponentials underflow and overflow, and of 0."""
    n = 401
    w = torch.zeros(2 * n, 2)
    w[:n, 0] = torch.arange(-200, 201).float()
    w[:n, 1] = 0
    w[n:, 1] = 1.0
    x = torch.ones(40, 2)
    q = i8.quantize(w.to(DEV))
    g, u = _sums(x, w)
    value, slope = ref.activation(np.clip(g, -700, 700), act)
    got = _np(i8.gated(x.to(DEV), q, activation=act))
    # below 2^-126 fp32's small numbers may be flushed
    assert (np.abs(got - value * u) <= np.abs(value * u) * _room(g) + 2.0 ** -120).all()
    dg = _np(i8.gated_gradient(torch.ones(40, n, device=DEV), x.to(DEV), q, activation=act))
    size = 1 / (1 + np.exp(-g)) * (1 + np.abs(g)) if act == "silu" else np.abs(slope) + np.abs(g) * np.exp(-g * g / 2)
    assert (np.abs(dg[:, :n] - slope * u) <= np.abs(u) * size * _room(g) + 2.0 ** -120).all()
    assert (np.abs(dg[:, n:] - value) <= np.abs(value) * _room(g) + 2.0 ** -120).all()


@pytest.mark.parametrize("rows,n_in,n", [(1, 5, 3), (33, 130, 70), (200, 300, 129)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_backward_is_the_layer_s_of_that_gradient(i8, rows, n_in, n, dtype):
    x, w, dh = _case(rows, n_in, n, dtype)
    q, qt = i8.quantize_both(w.to(DEV))
    x, dh = x.to(DEV), dh.to(DEV)
    for act in ("silu", "gelu"):
        dg = i8.gated_gradient(dh, x, q, activation=act)
        dx, dw = i8.gated_backward(dh, x, q, qt, activation=act)
        want = i8.linear_backward(dg, x, qt)
        assert dx.dtype == dtype and torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    base = torch.ones_like(dw)
    none, into = i8.gated_backward(dh, x, q, None, activation=act, dw=base, accumulate=True, need_dx=False)
    assert none is None and into is base and torch.equal(base, i8.linear_backward(dg, x, None, dw=torch.ones_like(dw), accumulate=True, need_dx=False)[1])


def test_a_token_of_no_numbers_stays_alone(i8):
    x, w, dh = _case(150, 200, 90, F32)
    x[70, 3] = float("nan")
    q, qt = i8.quantize_both(w.to(DEV))
    h = _np(i8.gated(x.to(DEV), q))
    assert np.isnan(h[70]).all() and np.isfinite(np.delete(h, 70, 0)).all()
    dx, dw = i8.gated_backward(dh.to(DEV), x.to(DEV), q, qt)
    assert np.isnan(_np(dx)[70]).all() and np.isfinite(np.delete(_np(dx), 70, 0)).all()
    assert np.isnan(_np(dw)).all()      # every column of dg holds that token

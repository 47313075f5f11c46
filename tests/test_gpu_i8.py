"""8-bit matrices, their products and layers: codes and results bit for bit against the definition, sizes and values where it can go wrong,
refusals, streams and graphs."""
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


def _x(rows, cols, dtype, seed, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen) * torch.exp(spread * torch.randn(rows, 1, generator=gen))
    return x.to(dtype)


def _np(x):
    return x.detach().float().cpu().numpy()


def _same_matrix(q, want, rows, cols):
    codes, scales, fine = want
    got = q.codes.cpu().numpy()
    pad = (cols + 127) // 128 * 128
    assert got.shape == (rows, pad) and (q.rows, q.cols) == (rows, cols)
    assert np.array_equal(got[:, :cols], np.where(fine[:, None], codes, 0))
    assert not got[:, cols:].any()
    assert np.array_equal(q.scales.cpu().numpy(), scales, equal_nan=True)


# a row in the registers of 1, 4 and 16 waves, and longer; columns in one run of rows and in many
SIZES = [(1, 1), (1, 7), (3, 128), (5, 129), (2, 2048), (7, 2049), (3, 8192), (2, 8193), (2, 40003), (63, 65), (64, 64), (129, 63), (300, 200), (2500, 70)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_codes_bit_for_bit(i8, rows, cols, dtype):
    x = _x(rows, cols, dtype, rows + cols)
    d = x.to(DEV)
    _same_matrix(i8.quantize(d), ref.integers(_np(x)), rows, cols)
    t = i8.quantize_columns(d)
    _same_matrix(t, ref.integers(_np(x).T), cols, rows)
    q, t2 = i8.quantize_both(d)
    assert torch.equal(q.codes, i8.quantize(d).codes) and torch.equal(t2.codes, t.codes) and torch.equal(t2.scales, t.scales)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first,more", [(0, 0), (1, 3), (3, 1), (8, 8)])
def test_rows_that_start_anywhere(i8, dtype, first, more):
    """A window of a larger matrix: strides and addresses that are no whole words; nothing around it is looked at."""
    rows, cols = 70, 260
    big = torch.full((rows, first + cols + more), float("nan"), dtype=dtype)
    big[:, first:first + cols] = _x(rows, cols, dtype, 5)
    x = big.to(DEV)[:, first:first + cols]
    want = _np(x)
    _same_matrix(i8.quantize(x), ref.integers(want), rows, cols)
    _same_matrix(i8.quantize_columns(x), ref.integers(want.T), cols, rows)


@pytest.mark.parametrize("rows", [255, 256, 257, 511, 512, 513, 1023, 1024, 1025])
@pytest.mark.parametrize("cols,first", [(77, 0), (264, 0), (2049, 0), (300, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_columns_of_few_and_of_many_rows(i8, rows, cols, first, dtype):
    gen = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols + 3, generator=gen).to(dtype)
    x[rows - 1, first] = float("inf")
    x[0, cols // 2] = float("nan")
    x[:, first + 2] = 0
    x = x.to(DEV)[:, first:first + cols]
    q, t = i8.quantize_both(x)
    want = ref.integers(_np(x).T)
    _same_matrix(q, ref.integers(_np(x)), rows, cols)
    _same_matrix(t, want, cols, rows)
    _same_matrix(i8.quantize_columns(x), want, cols, rows)


def test_columns_of_1024_rows_that_are_too_many_for_one_launch(i8):
    x = torch.randn(1024, 8200, generator=torch.Generator().manual_seed(5)).to(DEV)
    want = ref.integers(_np(x).T)
    _same_matrix(i8.quantize_columns(x), want, 8200, 1024)
    _same_matrix(i8.quantize_columns(x[:, :8192].contiguous()), tuple(v[:8192] for v in want), 8192, 1024)


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -20, 2.0 ** 100, 127.0 / 254])
def test_halves_go_to_the_even_integer(i8, scale):
    """Numbers half way between two integers, every one of them, and their neighbours on both sides."""
    half = np.arange(-127, 127) + 0.5
    x = np.concatenate([[127.0], half, np.arange(-127, 128)]).astype(np.float32) * np.float32(scale)
    x = np.stack([x, np.nextafter(x, np.float32(np.inf)), np.nextafter(x, np.float32(-np.inf))])
    x[:, 0] = np.float32(127) * np.float32(scale)
    _same_matrix(i8.quantize(torch.from_numpy(x).to(DEV)), ref.integers(x), *x.shape)
    _same_matrix(i8.quantize_columns(torch.from_numpy(np.ascontiguousarray(x.T)).to(DEV)), ref.integers(x), *x.shape)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_nothing_tiny_huge_and_no_numbers(i8, dtype):
    x = _x(8, 300, F32, 3)
    x[0] = 0
    x[1] *= 2.0 ** -110
    x[2] *= 2.0 ** -140
    x[3] = x[3] / x[3].abs().max() * 3.3e38
    x[4, 17] = float("nan")
    x[5, 299] = float("inf")
    x[6, 0] = -float("inf")
    x = x.to(dtype)
    _same_matrix(i8.quantize(x.to(DEV)), ref.integers(_np(x)), 8, 300)
    _same_matrix(i8.quantize_columns(x.to(DEV)), ref.integers(_np(x).T), 300, 8)
    w = i8.quantize(_x(40, 300, F32, 4).to(DEV))
    y = _np(i8.linear(x.to(DEV), w))
    assert np.isnan(y[4:7]).all() and np.isfinite(y[[0, 1, 2, 7]]).all() and not y[0].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (9, 127), (70, 260)])
def test_back_into_values(i8, rows, cols, dtype):
    x = _x(rows, cols, F32, 9)
    a = ref.integers(_np(x))
    want = torch.from_numpy(a[0].astype(np.float32) * a[1][:, None]).to(dtype)
    assert torch.equal(i8.dequantize(i8.quantize(x.to(DEV)), dtype).cpu(), want)


# one row and a few, tiles that are half empty, a sum of less than a step, of one, of many
PRODUCTS = [(1, 1, 1), (1, 1000, 700), (2, 17, 128), (3, 33, 129), (4, 256, 1000), (5, 100, 4096), (16, 16, 64), (17, 40, 5000), (33, 65, 300), (64, 64, 2500),
            (100, 200, 384), (128, 128, 128), (129, 257, 640), (300, 520, 1111), (700, 900, 256)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_bit_for_bit(i8, m, n, k, dtype):
    a, b = _x(m, k, F32, 1), _x(n, k, F32, 2)
    want = torch.from_numpy(ref.product(ref.integers(_np(a)), ref.integers(_np(b)))).to(dtype)
    qa, qb = i8.quantize(a.to(DEV)), i8.quantize(b.to(DEV))
    got = i8.matmul(qa, qb, dtype)
    assert torch.equal(got.cpu(), want)
    assert torch.equal(i8.linear(a.to(DEV), qb, dtype).cpu(), want)
    bf = a.to(BF16)
    want = torch.from_numpy(ref.product(ref.integers(_np(bf)), ref.integers(_np(b)))).to(dtype)
    assert torch.equal(i8.linear(bf.to(DEV), qb, dtype).cpu(), want)
    # into a window of a larger matrix, added to what is there: one more rounding, of the sum
    big = torch.full((m, n + 3), 7.0, dtype=dtype, device=DEV)
    i8.matmul(qa, qb, out=big[:, 1:n + 1], accumulate=True)
    more = (got.float() if dtype == F32 else i8.matmul(qa, qb, F32)) + 7.0
    # (the product with the scales and the sum may be one fused operation, which leaves the first rounding out)
    far = (big[:, 1:n + 1].float() - more).abs()
    assert (far <= ref.F32_HALF * 2 * (more.abs() + 7 + (more - 7).abs()) + (ref.BF16_HALF * more.abs() if dtype == BF16 else 0)).all()
    assert (big[:, 0] == 7).all() and (big[:, n + 1:] == 7).all()


def test_the_largest_sums(i8):
    """All codes 127, the longest sum: 2^17 x 127^2 fits 32 bits."""
    k = 131072
    a = torch.ones(3, k, device=DEV)
    a[1] = -1
    q = i8.quantize(a)
    want = ref.product(ref.integers(_np(a)), ref.integers(_np(a)))
    assert np.array_equal(_np(i8.matmul(q, q)), want)
    assert np.array_equal(_np(i8.linear(a, q)), want)


@pytest.mark.parametrize("rows,n_in,n_out", [(1, 5, 3), (7, 64, 33), (130, 300, 200), (257, 100, 513), (1000, 70, 130)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_a_layer_bit_for_bit(i8, rows, n_in, n_out, dtype):
    x, dy, w = _x(rows, n_in, dtype, 1), _x(rows, n_out, dtype, 2, 2.0), _x(n_out, n_in, F32, 3)
    wt = i8.quantize_columns(w.to(DEV))
    dx, dw = i8.linear_backward(dy.to(DEV), x.to(DEV), wt)
    want_dx = torch.from_numpy(ref.product(ref.integers(_np(dy)), ref.integers(_np(w).T))).to(dtype)
    want_dw = torch.from_numpy(ref.product(ref.integers(_np(dy).T), ref.integers(_np(x).T)))
    assert torch.equal(dx.cpu(), want_dx) and torch.equal(dw.cpu(), want_dw)
    none, dw2 = i8.linear_backward(dy.to(DEV), x.to(DEV), None, need_dx=False, dw_dtype=BF16)
    assert none is None and torch.equal(dw2.cpu(), want_dw.to(BF16))


def test_gradients_against_differences(i8):
    """y is linear in what the codes stand for: moving one weight by a whole number of steps moves a loss by what dw says, up to what
    quantising dy and x leaves out (half a step of 127 of their columns' largest for each factor)."""
    rows, n_in, n_out = 64, 48, 40
    x, w, c = _x(rows, n_in, F32, 1, 0.2), _x(n_out, n_in, F32, 2, 0.2), _x(rows, n_out, F32, 3, 0.2)
    q, qt = i8.quantize_both(w.to(DEV))
    dx, dw = i8.linear_backward(c.to(DEV), x.to(DEV), qt)
    xv, cv = _np(x).astype(np.float64), _np(c).astype(np.float64)
    qx = ref.values(ref.integers(_np(x)))
    for o, i in ((0, 0), (17, 30), (39, 47)):
        codes = q.codes.clone()
        step = 1 if codes[o, i] < 127 else -1
        codes[o, i] += step
        moved = i8.I8Matrix(codes, q.scales, n_out, n_in)
        change = ((_np(i8.linear(x.to(DEV), moved)).astype(np.float64) - _np(i8.linear(x.to(DEV), q))) * cv).sum()
        rate = change / (step * float(q.scales[o]))
        # both see quantised x, the difference by rows and dw by columns, and dw quantised dy
        room = np.abs(cv[:, o]).sum() * np.abs(xv).max() / 254 * 2 + np.abs(xv[:, i]).sum() * np.abs(cv[:, o]).max() / 254 * 1.1 + 1e-3 * np.abs(cv[:, o] * qx[:, i]).sum()
        assert abs(rate - float(dw[o, i])) <= room
    # dx against the formula's in float64
    wv = _np(w).astype(np.float64)
    room = np.abs(wv).sum(0)[None, :] * np.abs(cv).max(1)[:, None] / 254 + np.abs(cv).sum(1)[:, None] * np.abs(wv).max(0)[None, :] / 254 * 1.1
    assert (np.abs(_np(dx) - cv @ wv) <= room + 1e-5).all()


@pytest.mark.parametrize("rows,cols,dtype", [(4097, 8200, BF16), (2100, 8193, F32), (131, 140000, F32)])
def test_columns_of_what_no_cache_holds(i8, rows, cols, dtype):
    """Over 64 MB, where both passes go past the caches: rows of whole words and not."""
    x = (torch.randn(rows, cols, device=DEV) * torch.exp(torch.randn(cols, device=DEV))).to(dtype)
    m = x.float().abs().amax(0)
    most = torch.full_like(m, 127.0)
    q = i8.quantize_columns(x)
    assert torch.equal(q.scales, m / most)
    assert torch.equal(q.codes[:, :rows].double(), torch.round(x.t().double() * (most / m).double()[:, None]))
    assert not q.codes[:, rows:].any()


def test_sizes_of_zero(i8):
    w = i8.quantize(torch.randn(6, 10, device=DEV))
    assert i8.linear(torch.empty(0, 10, device=DEV), w).shape == (0, 6)
    nothing = i8.quantize(torch.empty(6, 0, device=DEV))
    assert not i8.linear(torch.empty(4, 0, device=DEV), nothing).any()
    assert not i8.gated(torch.empty(4, 0, device=DEV), nothing).any()
    assert i8.linear(torch.randn(4, 10, device=DEV), i8.quantize(torch.empty(0, 10, device=DEV))).shape == (4, 0)
    dx, dw = i8.linear_backward(torch.empty(0, 6, device=DEV), torch.empty(0, 10, device=DEV), i8.quantize_columns(torch.randn(6, 10, device=DEV)))
    assert dx.shape == (0, 10) and dw.shape == (6, 10) and not dw.any()
    dx, dw = i8.linear_backward(torch.empty(5, 0, device=DEV), torch.randn(5, 10, device=DEV), i8.quantize(torch.empty(10, 0, device=DEV)))
    assert not dx.any() and dw.shape == (0, 10)
    dw = torch.ones(6, 10, device=DEV)
    i8.linear_backward(torch.empty(0, 6, device=DEV), torch.empty(0, 10, device=DEV), None, need_dx=False, dw=dw, accumulate=True)
    assert (dw == 1).all()


def test_refusals(i8):
    x, w = torch.randn(4, 10, device=DEV), i8.quantize(torch.randn(6, 10, device=DEV))
    for call in (lambda: i8.linear(x[:, :9], w), lambda: i8.linear(x.t(), w), lambda: i8.linear(x.cpu(), w), lambda: i8.linear(x[0], w),
                 lambda: i8.linear(x, w._replace(scales=w.scales.double())), lambda: i8.linear(x, w._replace(codes=w.codes[:, :64])),
                 lambda: i8.linear(x.clone().requires_grad_(), w), lambda: i8.matmul(w, w, accumulate=True),
                 lambda: i8.matmul(w, w, out=torch.empty(6, 5, device=DEV)), lambda: i8.gated(x, i8.quantize(torch.randn(5, 10, device=DEV))),
                 lambda: i8.gated(x, w, activation="tanh"), lambda: i8.linear_backward(torch.randn(3, 6, device=DEV), x, w),
                 lambda: i8.linear_backward(torch.randn(4, 6, device=DEV), x.bfloat16(), w), lambda: i8.gated(x.clone().requires_grad_(), w),
                 lambda: i8.gated_gradient(torch.randn(4, 4, device=DEV), x, w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        i8.linear(x.half(), w)
    with torch.no_grad():
        assert torch.equal(i8.linear(x.clone().requires_grad_(), w), i8.linear(x, w))


def test_another_stream_and_graphs(i8):
    x, w = _x(300, 260, F32, 1).to(DEV), _x(140, 260, F32, 2).to(DEV)
    dy, dh = _x(300, 140, F32, 3).to(DEV), _x(300, 70, F32, 4).to(DEV)
    q, qt = i8.quantize_both(w)

    def all_of_it():
        return [i8.linear(x, q), i8.linear(x[:2], q), i8.gated(x, q), i8.gated(x[:1], q), *i8.linear_backward(dy, x, qt), i8.gated_gradient(dh, x, q),
                *i8.gated_backward(dh, x, q, qt), i8.quantize_columns(x).codes]
    want = all_of_it()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = all_of_it()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(all_of_it())
        graphs.append(g)
    for turn in range(4):
        x.mul_(1.5)
        dy.add_(0.25)
        want = all_of_it()
        for g in graphs[::1 if turn % 2 else -1]:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(want, out)), turn

"""4-bit microscaled matrices, their products and layers against float64 from the definition.

Codes and scales are whole numbers and have to be equal.  A product sums K exact products in fp32, 128 of them per matrix instruction:
K / 128 + 2 roundings of at most 2^-22 (twice an fp32 rounding, for sums inside the instruction that may be cut off) of the sum of
magnitudes; a bf16 result adds half a unit of its last place, 2^-8.
"""
import numpy as np
import pytest

import _mx_reference as ref
from paper_1811_03617_amd import gvq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def mx():
    from paper_1811_03617_amd import mx
    return mx


def _host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _numbers(rows, cols, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(spread * torch.randn(1, cols, generator=g))
    # ties, zeros, numbers that round to 6 from above, and whole blocks of zeros
    if rows and cols:
        x[rows // 2] = torch.round(x[rows // 2] * 4) / 4
        x[0, : min(cols, 40)] = 0.0
    return x.to(dtype).to(DEV)


def _noise(rows, cols, seed):
    return torch.randint(0, 256, (rows, cols), generator=torch.Generator().manual_seed(seed), dtype=torch.uint8).to(DEV)


def _same(q, x, noise=None):
    code, scale = ref.encode(x, noise)
    assert np.array_equal(q.scales.cpu().numpy().reshape(scale.shape), scale)
    # the sign of a number that rounds to 0 is kept; behind the last column there is nothing
    assert np.array_equal(q.codes.cpu().numpy(), ref.pack(code))


SIZES = [(1, 1), (1, 31), (1, 32), (1, 33), (3, 127), (5, 128), (2, 129), (31, 64), (32, 257), (33, 96), (127, 65), (128, 128), (129, 200),
         (260, 333), (1, 4096), (37, 4096)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("noisy", [False, True])
def test_quantize_both_directions_is_exact(mx, rows, cols, dtype, noisy):
    x = _numbers(rows, cols, dtype, rows * 1000 + cols)
    z = _noise(rows, cols, cols) if noisy else None
    xh, zh = _host(x), None if z is None else z.cpu().numpy().astype(np.float64)
    q, t = mx.quantize_both(x, z)
    _same(q, xh, zh)
    _same(t, xh.T, None if zh is None else zh.T)
    for one, two in ((mx.quantize(x, z), q), (mx.quantize_columns(x, z), t)):
        assert torch.equal(one.codes, two.codes) and torch.equal(one.scales, two.scales)
    for got, want in ((q, xh), (t, xh.T)):
        w = ref.quantized(want, zh if got is q else None if zh is None else zh.T)
        assert np.array_equal(_host(mx.dequantize(got)), w)
        assert np.array_equal(_host(mx.dequantize(got, torch.bfloat16)), w)


def test_quantize_every_bf16_number(mx):
    """Each finite bf16 number beside every power of two from 4 times smaller on: all roundings, ties, denormals and scales."""
    bits = np.arange(0, 0x7F80, dtype=np.uint16)
    f = (bits.astype(np.uint32) << 16).view(np.float32)
    rows = []
    for up in (0, 1, 2, 3, 4):
        block = np.zeros((f.size, 32), np.float32)
        block[:, 0] = f
        block[:, 1] = -f
        with np.errstate(over="ignore"):
            block[:, 2] = np.minimum(f * np.float32(2.0 ** up), np.float32(3.0e38))
        rows.append(block)
    x = torch.from_numpy(np.concatenate(rows)).to(torch.bfloat16)
    xh = _host(x)
    for dt in (torch.bfloat16, torch.float32):
        _same(mx.quantize(x.to(dt).to(DEV)), xh)


def test_quantize_extremes(mx):
    inf, nan, tiny, big = float("inf"), float("nan"), 1.4e-45, 3.4028234e38
    x = torch.zeros(12, 96)
    x[0, 5] = inf
    x[1, 40] = -inf
    x[2, 95] = nan
    x[3, 0], x[3, 1] = tiny, -tiny
    x[4, 7], x[4, 8] = big, -big / 3
    x[5] = 1e-39                       # denormals
    x[6, ::2] = 6.0
    x[6, 1::2] = 7.99
    x[7] = -0.0
    x[8, 3] = 2.0 ** -126
    x[9, 3], x[9, 4] = 2.0 ** -124, 2.0 ** -126
    x[10, 33], x[10, 34] = inf, 1.0
    x[11] = 2.0 ** -149
    for z in (None, torch.full((12, 96), 255, dtype=torch.uint8), torch.zeros(12, 96, dtype=torch.uint8)):
        zd = None if z is None else z.to(DEV)
        zh = None if z is None else z.numpy().astype(np.float64)
        q, t = mx.quantize_both(x.to(DEV), zd)
        xh = x.double().numpy()
        _same(q, xh, zh)
        _same(t, xh.T, None if zh is None else zh.T)
        back = _host(mx.dequantize(q))
        assert np.array_equal(back, ref.quantized(xh, zh), equal_nan=True)
    assert np.isnan(back[0, :32]).all() and np.array_equal(back[0, 32:], np.zeros(64))


def test_quantize_strided_and_unaligned(mx):
    big = _numbers(70, 300, torch.float32, 5)
    zbig = _noise(70, 300, 6)
    for dt in (torch.float32, torch.bfloat16):
        b = big.to(dt)
        for view, z in ((b[:, 3:200], zbig[:, 3:200]), (b[1::2, 8:136], zbig[1::2, 8:136]), (b[5:6, 1:], zbig[5:6, 1:])):
            q, t = mx.quantize_both(view, z)
            _same(q, _host(view), z.cpu().numpy().astype(np.float64))
            _same(t, _host(view).T, z.cpu().numpy().T.astype(np.float64))
            out = torch.full((view.shape[0], view.shape[1] + 5), 7.0, dtype=dt, device=DEV)
            gvq.gvq_mx_dequantize(q.codes, q.scales, q.rows, q.cols, out[:, 1:], gvq.F32 if dt == torch.float32 else gvq.BF16, out.shape[1])
            assert torch.equal(out[:, 1:-4], mx.dequantize(q, dt)) and bool((out[:, :1] == 7).all()) and bool((out[:, -4:] == 7).all())


def test_stochastic_rounding_is_unbiased(mx):
    """Over all 256 bytes a number 1/256 n + 1/512 of the way up goes up n + 0 or 1 times: the mean is within 1/512 of a step."""
    v = torch.linspace(-5.9, 5.9, 301)
    x = torch.zeros(256, 320)
    x[:, :301] = v
    x[:, 31::32] = 6.0                  # every block's scale is 1
    z = torch.arange(256, dtype=torch.uint8)[:, None].expand(256, 320).contiguous()
    got = _host(mx.dequantize(mx.quantize(x.to(DEV), z.to(DEV)))).mean(0)
    step = np.where(np.abs(x[0].numpy()) < 2, 0.5, np.where(np.abs(x[0].numpy()) < 4, 1.0, 2.0))
    # fp32 numbers of the grid's size: an exact mean, compared with the number as fp32 holds it
    assert np.all(np.abs(got - x[0].double().numpy()) <= step / 512 + 1e-12)


def _random_mx(mx, rows, cols, seed, spread=1.0):
    x = _numbers(rows, cols, torch.float32, seed, spread)
    q = mx.quantize(x)
    return q, ref.quantized(_host(x))


def _product_bound(a, b, dtype):
    mag = np.abs(a) @ np.abs(b).T
    k = a.shape[1]
    tol = (k / 128 + 2) * 2.0 ** -22 * mag
    return tol + (np.abs(a @ b.T) * 2.0 ** -8 if dtype == torch.bfloat16 else 0)


PRODUCTS = [(1, 1, 1), (1, 17, 33), (16, 16, 128), (17, 63, 129), (5, 1000, 640), (64, 64, 256), (65, 65, 384), (130, 70, 1000), (300, 260, 512),
            (1, 300, 4096), (15, 513, 2048), (33, 129, 900), (128, 192, 2100), (513, 1030, 200)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matmul(mx, m, n, k, dtype):
    a, ah = _random_mx(mx, m, k, 1 + m)
    b, bh = _random_mx(mx, n, k, 2 + n)
    want, tol = ah @ bh.T, _product_bound(ah, bh, dtype)
    got = mx.matmul(a, b, dtype)
    assert np.all(np.abs(_host(got) - want) <= tol)
    # into a strided, unaligned place, and added to it
    big = torch.full((m, n + 9), 0.25, dtype=dtype, device=DEV)
    for view in (big[:, 1:n + 1], big[:, 4:n + 4]):
        view.fill_(0.25)
        mx.matmul(a, b, out=view)
        assert torch.equal(view, got)
        mx.matmul(a, b, out=view, accumulate=True)
        twice = _host(got) + want
        assert np.all(np.abs(_host(view) - twice) <= 2 * tol + (np.abs(twice) * 2.0 ** -8 if dtype == torch.bfloat16 else np.abs(twice) * 2.0 ** -23))
        view.fill_(0.25)
        assert bool((big == 0.25).all())


@pytest.mark.parametrize("m,n,k", [(3300, 4224, 300), (2080, 6200, 160)])
def test_matmul_many_tiles(mx, m, n, k):
    """Grids of the largest tiles with ragged last ones; whole numbers, so fp32 sums are exact."""
    g = torch.Generator().manual_seed(m)
    a, b = (torch.randint(-6, 7, s, generator=g).float().to(DEV) for s in ((m, k), (n, k)))
    qa, qb = mx.quantize(a), mx.quantize(b)
    want = mx.dequantize(qa).double() @ mx.dequantize(qb).double().t()
    assert torch.equal(mx.matmul(qa, qb).double(), want)


def test_products_keep_nan_in_its_rows_and_columns(mx):
    x = _numbers(70, 256, torch.float32, 3)
    w = _numbers(40, 256, torch.float32, 4)
    x[7, 100] = float("nan")
    w[11, 3] = float("inf")
    for y in (mx.linear(x, mx.quantize(w)), mx.linear(x[:9].contiguous(), mx.quantize(w))):
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[7] = True
        bad[:, 11] = True
        assert torch.equal(torch.isnan(y), bad)


LAYERS = [(1, 64, 10), (1, 25088, 48), (2, 100, 33), (7, 129, 65), (16, 512, 100), (17, 512, 100), (40, 4096, 64), (77, 640, 1000), (150, 300, 70),
          (300, 1056, 520)]


@pytest.mark.parametrize("rows,n_in,n_out", LAYERS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_linear_forward_and_backward(mx, rows, n_in, n_out, dtype):
    x = _numbers(rows, n_in, dtype, rows)
    w = _numbers(n_out, n_in, torch.float32, n_out)
    dy = _numbers(rows, n_out, dtype, 9)
    z = _noise(rows, n_out, 10)
    q, qt = mx.quantize_both(w)
    xh, wh, dyh, zh = _host(x), _host(w), _host(dy), z.cpu().numpy().astype(np.float64)
    a, b = ref.quantized(xh), ref.quantized(wh)
    for dt in (None, torch.float32):
        got = mx.linear(x, q, dt)
        assert got.dtype == (dt or dtype)
        assert np.all(np.abs(_host(got) - a @ b.T) <= _product_bound(a, b, got.dtype))
    for noise, n in ((None, None), (z, zh)):
        d, t = ref.quantized(dyh, n), ref.quantized(wh.T)
        dt, xt = ref.quantized(dyh.T, None if n is None else n.T), ref.quantized(xh.T)
        dx, dw = mx.linear_backward(dy, x, qt, noise=noise)
        assert dx.dtype == dtype and dw.dtype == torch.float32
        assert np.all(np.abs(_host(dx) - d @ t.T) <= _product_bound(d, t, dtype))
        assert np.all(np.abs(_host(dw) - dt @ xt.T) <= _product_bound(dt, xt, torch.float32))
        none, dw2 = mx.linear_backward(dy, x, None, noise=noise, need_dx=False)
        assert none is None and torch.equal(dw, dw2)
        more = dw.clone()
        mx.linear_backward(dy, x, qt, noise=noise, dw=more, accumulate=True)
        assert np.all(np.abs(_host(more) - 2 * (dt @ xt.T)) <= 3 * _product_bound(dt, xt, torch.float32))


def test_linear_gradients_against_differences(mx):
    """Inputs that 4 bits hold exactly: the layer is linear there, and differences of the loss sum(y c) over a step of the grid are its
    gradient exactly."""
    g = torch.Generator().manual_seed(1)
    R, K, N = 33, 64, 40
    # magnitudes of the grid, with 6 in every block along both axes: every scale is 1
    pick = torch.tensor([0.0, 0.5, 1.0, 2.0, 3.0, 4.0, 6.0])
    def grid(r, c):
        t = pick[torch.randint(0, 7, (r, c), generator=g)] * (torch.randint(0, 2, (r, c), generator=g) * 2 - 1)
        t[::16] = 6.0
        t[:, ::16] = 6.0
        return t.to(DEV)
    x, w, c = grid(R, K), grid(N, K), grid(R, N)
    q, qt = mx.quantize_both(w)
    dx, dw = mx.linear_backward(c, x, qt)
    loss = lambda x, q: (mx.linear(x, q).double() * c.double()).sum().item()
    base = loss(x, q)
    for i, j in ((1, 1), (20, 37), (31, 63)):
        p = x.clone()
        p[i, j] = 1.5 if p[i, j] != 1.5 else 1.0
        assert loss(p, q) - base == pytest.approx((dx[i, j] * (p[i, j] - x[i, j])).item(), rel=1e-6, abs=1e-3)
        v = w.clone()
        v[i, j] = 1.5 if v[i, j] != 1.5 else 1.0
        assert loss(x, mx.quantize(v)) - base == pytest.approx((dw[i, j] * (v[i, j] - w[i, j])).item(), rel=1e-6, abs=1e-3)


def test_empty_sizes(mx):
    for r, c in ((0, 64), (5, 0), (0, 0)):
        x = torch.zeros(r, c, device=DEV)
        q, t = mx.quantize_both(x)
        assert mx.dequantize(q).shape == (r, c) and mx.dequantize(t).shape == (c, r)
    w = mx.quantize(_numbers(20, 64, torch.float32, 1))
    assert mx.linear(torch.zeros(0, 64, device=DEV), w).shape == (0, 20)
    none = mx.quantize(torch.zeros(20, 0, device=DEV))
    assert torch.equal(mx.linear(torch.zeros(3, 0, device=DEV), none), torch.zeros(3, 20, device=DEV))
    dx, dw = mx.linear_backward(torch.zeros(0, 20, device=DEV), torch.zeros(0, 64, device=DEV), mx.quantize(torch.ones(64, 20, device=DEV)))
    assert dx.shape == (0, 64) and torch.equal(dw, torch.zeros(20, 64, device=DEV))
    keep = torch.ones(20, 64, device=DEV)
    mx.linear_backward(torch.zeros(0, 20, device=DEV), torch.zeros(0, 64, device=DEV), None, dw=keep, accumulate=True, need_dx=False)
    assert torch.equal(keep, torch.ones(20, 64, device=DEV))


def test_other_streams_and_repeats(mx):
    x, w = _numbers(200, 1000, torch.bfloat16, 1), _numbers(300, 1000, torch.float32, 2)
    q = mx.quantize(w)
    want = mx.linear(x, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [mx.linear(x, mx.quantize(w)) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_graph_replays(mx):
    x, w, dy = _numbers(100, 256, torch.bfloat16, 1), _numbers(90, 256, torch.float32, 2), _numbers(100, 90, torch.bfloat16, 3)
    def work():
        q, qt = mx.quantize_both(w)
        return (mx.linear(x, q), mx.linear(x[:3], q)) + mx.linear_backward(dy, x, qt)
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for k in range(3):
        x.copy_(_numbers(100, 256, torch.bfloat16, 20 + k))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, work()):
            assert torch.equal(a, b)


def test_refusals(mx):
    L = gvq.lib()
    st = torch.cuda.current_stream().cuda_stream
    x = torch.zeros(8, 64, device=DEV)
    q = mx.quantize(x)
    c, s, p = q.codes.data_ptr(), q.scales.data_ptr(), x.data_ptr()
    quant = L.gvq_mx_quantize
    assert quant(p, gvq.F32, 8, 64, 63, None, 0, c, s, None, None, st) == gvq.EINVAL
    assert quant(p, 7, 8, 64, 64, None, 0, c, s, None, None, st) == gvq.EINVAL
    assert quant(p, gvq.F32, -1, 64, 64, None, 0, c, s, None, None, st) == gvq.EINVAL
    assert quant(p, gvq.F32, 8, gvq.MX_MAX + 1, gvq.MX_MAX + 1, None, 0, c, s, None, None, st) == gvq.EINVAL
    assert quant(p, gvq.F32, 8, 64, 64, None, 0, None, None, None, None, st) == gvq.EINVAL
    assert quant(p, gvq.F32, 8, 64, 64, None, 0, c, None, None, None, st) == gvq.EINVAL
    assert quant(None, gvq.F32, 8, 64, 64, None, 0, c, s, None, None, st) == gvq.EINVAL
    assert quant(p, gvq.F32, 8, 64, 64, p, 60, c, s, None, None, st) == gvq.EINVAL
    assert quant(p, gvq.F32, 8, 64, 64, None, 0, c + 4, s, None, None, st) == gvq.EALIGN
    assert quant(p + 2, gvq.F32, 8, 64, 64, None, 0, c, s, None, None, st) == gvq.EALIGN
    assert L.gvq_mx_dequantize(c, s, 8, 64, p, gvq.F32, 60, st) == gvq.EINVAL
    assert L.gvq_mx_dequantize(c, None, 8, 64, p, gvq.F32, 64, st) == gvq.EINVAL
    assert L.gvq_mx_matmul(c, s, c, s, 8, 8, 64, p, gvq.F32, 7, 0, st) == gvq.EINVAL
    assert L.gvq_mx_matmul(c, s, c, None, 8, 8, 64, p, gvq.F32, 8, 0, st) == gvq.EINVAL
    assert L.gvq_mx_matmul(c + 8, s, c, s, 8, 8, 64, p, gvq.F32, 8, 0, st) == gvq.EALIGN
    assert L.gvq_mx_linear(p, gvq.F32, 8, 64, 64, c, s, 8, p, gvq.F32, 8, None, st) == gvq.EINVAL
    assert L.gvq_mx_linear_backward(p, 8, p, 64, gvq.F32, 8, 64, 8, None, 0, c, s, None, 0, 0, None, 0, 0, 0, p, st) == gvq.EINVAL
    with pytest.raises(TypeError):
        mx.quantize(x.half())
    with pytest.raises(ValueError):
        mx.quantize(x.t())
    with pytest.raises(ValueError):
        mx.quantize(x, noise=torch.zeros(8, 63, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        mx.quantize(x.cpu())
    with pytest.raises(ValueError):
        mx.linear(torch.zeros(2, 65, device=DEV), q)
    with pytest.raises(ValueError):
        mx.matmul(q, q, accumulate=True)
    with pytest.raises(ValueError):
        mx.matmul(q, q._replace(codes=q.codes[:4]))
    with pytest.raises(ValueError):
        mx.linear_backward(torch.zeros(3, 8, device=DEV), torch.zeros(4, 64, device=DEV), q)

"""8-bit products through each of the ways they can take: straight from memory (16 or 32 rows a work-group, few of these in numbers) and tiles of
three shapes, the smallest with sums of one team, two and four; one product and two in one launch; plain, gated, and the gated block's inner gradient.

Whole numbers of up to 127 with 127 in every row: each scale is 1 and a sum is exact, so that a plain result is that sum rounded once.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16

# rows of A and B, numbers of the sum; none of them whole tiles
PLAIN = [
    (17, 300, 900), (9, 70, 12500), (40, 1000, 700),        # 16 rows a work-group
    (17, 4096, 4097), (77, 1000, 4096),                     # 32
    (500, 1001, 300), (100, 4099, 384), (129, 2500, 250),   # tiles: 64 x 64
    (50, 6801, 700), (80, 3409, 1500), (80, 3409, 129),     # their sums by two teams
    (65, 4096, 16300), (300, 2500, 4096),                   # and by four
    (1000, 8190, 2000),                                     # 128 x 128
    (3000, 4097, 520), (2049, 8190, 1300),                  # 256 x 256
]
GATED = [
    (17, 300, 900), (9, 70, 12500),
    (17, 3409, 300), (30, 3409, 700),
    (500, 1001, 300), (129, 2500, 250),
    (17, 6801, 700), (300, 2500, 4096),
    (17, 4096, 4097), (77, 1000, 4096),
    (444, 6801, 700), (293, 3409, 6300),
    (600, 8001, 1000), (2049, 4100, 130),
]
# rows, columns in and out of a layer
PAIRS = [
    (33, 130, 70), (300, 261, 140), (257, 100, 513),        # both gradients in one launch: 64 x 64
    (1000, 1000, 1000),                                     # two teams
    (1521, 123, 3100), (1521, 70, 6300),                    # four
    (500, 4096, 1000),
    (2000, 3001, 2500),
    (2286, 3409, 3100),                                     # a launch each
]


@pytest.fixture(scope="module")
def i8():
    from paper_1811_03617_amd import i8 as module
    return module


def _whole(rows, cols, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randint(-127, 128, (rows, cols), generator=g, device=DEV).float()
    x[:, seed % cols] = 127.0
    return x


def _sums(a, b):
    return a.double() @ b.double().t().contiguous()


@pytest.mark.parametrize("m,n,k", PLAIN)
def test_products_of_whole_numbers(i8, m, n, k):
    a, b = _whole(m, k, m), _whole(n, k, n)
    qa, qb = i8.quantize(a), i8.quantize(b)
    assert (qa.scales == 1).all() and (qb.scales == 1).all()
    want = _sums(a, b).float()
    assert torch.equal(i8.matmul(qa, qb), want)
    assert torch.equal(i8.matmul(qa, qb, BF16), want.to(BF16))
    # in rows that start anywhere, and added to what is there: a power of two far above, so that no bit is lost
    for dtype in (F32, BF16):
        place = torch.full((m, n + 5), 0.5, dtype=dtype, device=DEV)
        view = place[:, 1:n + 1]
        i8.matmul(qa, qb, out=view)
        assert torch.equal(view, want.to(dtype))
        i8.matmul(qa, qb, out=view, accumulate=True)
        assert torch.equal(view, (want.to(dtype).float() + want).to(dtype))
        view.fill_(0.5)
        assert bool((place == 0.5).all())


@pytest.mark.parametrize("m,n,k", GATED)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_blocks_of_whole_numbers(i8, m, n, k, dtype):
    """Every place's g and u are the ones of its row and column: weights are scaled down so that neighbours' differ by far more than the
    activation's rounding (which test_gpu_gated.py holds to its own bound)."""
    x, w = _whole(m, k, m).to(dtype), _whole(2 * n, k, n + 1)
    q = i8.quantize(w)
    q = q._replace(scales=q.scales * (4.0 / (127 * k ** 0.5)) ** 2)   # sums of the order of 1
    s = _sums(x, w).float() * q.scales[None, :]
    g, u = s[:, :n].double(), s[:, n:].double()
    sig = torch.sigmoid(g)
    last = 2.0 ** -8 if dtype == BF16 else 0.0
    want = g * sig * u
    got = i8.gated(x, q).double()
    assert ((got - want).abs() <= want.abs() * (last + 2.0 ** -24 * (60 + 8 * g.abs()))).all()
    dh = _whole(m, n, 7).to(dtype) / 64
    d = dh.double()
    got = i8.gated_gradient(dh, x, q).double()
    slope = sig * (1 + g * (1 - sig))
    room = 2.0 ** -24 * (60 + 8 * g.abs())
    assert ((got[:, :n] - d * u * slope).abs() <= (d * u).abs() * (slope.abs() * last + sig * (1 + g.abs()) * room) * (1 + last)).all()
    assert ((got[:, n:] - d * g * sig).abs() <= (d * g * sig).abs() * (last + room) * (1 + last)).all()


@pytest.mark.parametrize("rows,n_in,n_out", PAIRS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_both_gradients_of_whole_numbers(i8, rows, n_in, n_out, dtype):
    x, dy, w = _whole(rows, n_in, 1), _whole(rows, n_out, 2), _whole(n_out, n_in, 3)
    # a largest number in every column too
    x[5 % rows] = 127.0
    dy[7 % rows] = -127.0
    w[3 % n_out] = 127.0
    qt = i8.quantize_columns(w)
    assert (qt.scales == 1).all()
    dx, dw = i8.linear_backward(dy.to(dtype), x.to(dtype), qt)
    assert torch.equal(dx, _sums(dy, w.t()).float().to(dtype))
    assert torch.equal(dw, _sums(dy.t(), x.t()).float())
    place = torch.ones(n_out, n_in + 3, device=DEV)[:, 2:n_in + 2]
    none, dw2 = i8.linear_backward(dy.to(dtype), x.to(dtype), None, need_dx=False, dw=place)
    assert torch.equal(dw2, dw)


# one to five rows, to few and to many columns: quantised by the product itself and by a launch of their own
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("n_in,n_out", [(100, 130), (700, 130), (12500, 33), (4097, 2000), (1000, 25089), (70000, 50)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layers_of_few_rows(i8, rows, n_in, n_out, dtype):
    x, w = _whole(rows, n_in, 3), _whole(n_out, n_in, 4)
    q = i8.quantize(w)
    want = _sums(x, w).float()
    for step in (n_in, n_in + 8 - n_in % 8, n_in + 1):   # rows that start at whole words, and do not
        p = torch.zeros(rows, step, dtype=dtype, device=DEV)[:, :n_in]
        p.copy_(x)
        assert torch.equal(i8.linear(p, q, F32), want)
    if n_out % 2 == 0:
        q = q._replace(scales=q.scales * (4.0 / (127 * n_in ** 0.5)) ** 2)
        s = (want * q.scales[None, :]).double()
        g, u = s[:, :n_out // 2], s[:, n_out // 2:]
        h = i8.gated(p, q, dtype=F32).double()
        assert ((h - g * torch.sigmoid(g) * u).abs() <= (g * torch.sigmoid(g) * u).abs() * 2.0 ** -24 * (60 + 8 * g.abs())).all()


def test_infinities_stay_in_their_row(i8):
    """Tokens that hold no numbers, through every way's rows, and a channel of no numbers."""
    for m, n, k in ((3, 100, 500), (17, 300, 900), (77, 1000, 4096), (129, 2500, 250), (300, 2500, 4096), (2049, 4100, 130)):
        x, w = _whole(m, k, 1), _whole(n, k, 2)
        x[m // 2, 3] = float("inf")
        w[n // 3, 5] = float("nan")
        y = i8.linear(x, i8.quantize(w))
        bad = torch.isnan(y)
        assert bad[m // 2].all() and bad[:, n // 3].all() and int(bad.sum()) == m + n - 1

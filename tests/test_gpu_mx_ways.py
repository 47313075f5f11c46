"""4-bit products through each of the ways they can take: without LDS (16 or 32 rows a work-group, few of these) and tiles of four shapes.

Whole numbers of the 4-bit grid with magnitudes up to 6: every sum is a whole number below 2^24, which fp32 holds exactly in any order
(36 x 12500 at most), and a bf16 result is that sum rounded once.  The two sides have to be equal.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rows of A and B, numbers of the sum; none of them whole tiles
SIZES = [
    (17, 300, 900), (31, 70, 12500), (40, 1000, 700), (130, 300, 5000),                        # 16 rows a work-group
    (17, 4096, 500), (77, 1000, 4096), (130, 530, 5000), (200, 515, 600),                      # 32
    (600, 2000, 3001), (49, 4100, 1000), (31, 20000, 5000),                                    # tiles: 64 x 64
    (17, 25090, 520), (1001, 4097, 500), (600, 900, 640),                                      # 128 x 128
    (130, 25000, 1100), (1500, 2900, 520),                                                     # 256 x 128
    (4000, 4090, 5000),                                                                        # 256 x 256
    (3, 9000, 300), (4, 25088, 300),                                                           # steps of the sum too few for the others
]


@pytest.fixture(scope="module")
def mx():
    from paper_1811_03617_amd import mx
    return mx


def _whole(rows, cols, seed):
    grid = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0])
    g = torch.Generator().manual_seed(seed)
    x = grid[torch.randint(0, 6, (rows, cols), generator=g)] * (torch.randint(0, 2, (rows, cols), generator=g) * 2 - 1)
    x[:, ::32] = 6.0   # every block's scale is 1
    return x.to(DEV)


@pytest.mark.parametrize("m,n,k", SIZES)
def test_products_of_whole_numbers(mx, m, n, k):
    a, b = _whole(m, k, m), _whole(n, k, n + 1)
    qa, qb = mx.quantize(a), mx.quantize(b)
    want = a.double() @ b.double().t().contiguous()
    assert torch.equal(mx.matmul(qa, qb).double(), want)
    assert torch.equal(mx.matmul(qa, qb, torch.bfloat16), want.float().to(torch.bfloat16))
    # in rows that start anywhere, and twice
    place = torch.full((m, n + 5), 0.5, device=DEV)
    view = place[:, 1:n + 1]
    mx.matmul(qa, qb, out=view)
    assert torch.equal(view.double(), want)
    mx.matmul(qa, qb, out=view, accumulate=True)
    assert torch.equal(view.double(), 2 * want)
    view.fill_(0.5)
    assert bool((place == 0.5).all())


# one to five rows, to few and to many columns: quantised by the product itself and by a launch of their own
@pytest.mark.parametrize("rows", [1, 2, 4, 5])
@pytest.mark.parametrize("n_in,n_out", [(700, 130), (12500, 33), (4097, 2000), (1000, 25089)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_layers_of_few_rows(mx, rows, n_in, n_out, dtype):
    x, w = _whole(rows, n_in, 3), _whole(n_out, n_in, 4)
    q = mx.quantize(w)
    want = x.double() @ w.double().t().contiguous()
    for step in (n_in, n_in + 8 - n_in % 8, n_in + 1):   # rows that start at whole words, and do not
        p = torch.zeros(rows, step, dtype=dtype, device=DEV)[:, :n_in]
        p.copy_(x)
        assert torch.equal(mx.linear(p, q, torch.float32).double(), want)

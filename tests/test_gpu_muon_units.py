"""Newton-Schulz at the ends of what its numbers can hold: norms far below eps, coefficients that let X grow, rows far smaller than others.

Tolerance of a whole matrix as in test_gpu_muon.py: 2e-5 of the 2-norm.
"""
import numpy as np
import pytest

from paper_1811_03617_amd import gvq  # noqa: F401  (the library itself)
from test_gpu_muon import DEFAULT, DEV, TOL, _exact, _host, _off

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32 = TOL[torch.float32]

# one launch; runs of columns, wide and tall; tiles, wide, tall and with the sum in parts
SIZES = [(40, 60), (27, 64), (64, 2000), (1000, 40), (130, 300), (300, 130), (128, 4608)]


@pytest.fixture(scope="module")
def muon():
    from paper_1811_03617_amd import muon
    return muon


def _of_norm(rows, cols, norm, seed):
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
    return (x * (norm / x.norm())).float().to(DEV)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("norm", [1e-6, 1e-7, 3e-8, 1e-9, 1e-11, 1e-13, 1e-20, 1e-30])
def test_norms_around_and_far_below_eps(muon, rows, cols, norm):
    """X is as small as the norm is beside eps: it is still as exact as any other."""
    g = _of_norm(rows, cols, norm, rows)
    assert _off(muon.orthogonalize(g), _exact(_host(g))) <= F32
    assert _off(muon.orthogonalize(g, steps=1), _exact(_host(g), DEFAULT[:1])) <= F32


@pytest.mark.parametrize("rows,cols", [(30, 50), (64, 700), (100, 160)])
def test_norms_of_a_batch_do_not_meet(muon, rows, cols):
    g = torch.stack([_of_norm(rows, cols, n, k) for k, n in enumerate([1.0, 1e-12, 1e-7, 0.0, 1e-25])])
    got = muon.orthogonalize(g)
    for k in range(len(g)):
        assert torch.equal(got[k], muon.orthogonalize(g[k].contiguous()))


@pytest.mark.parametrize("rows,cols", [(30, 50), (64, 700), (160, 100)])
def test_steps_of_a_tiny_momentum(muon, rows, cols):
    g, m, w = _of_norm(rows, cols, 1e-12, 1), _of_norm(rows, cols, 2e-12, 2), _of_norm(rows, cols, 1e-4, 3)
    mh = 0.9 * _host(m) + _host(g)
    o = _exact(_host(g) + 0.9 * mh)
    want = _host(w) - 0.1 * o
    muon.step(w, g, m, lr=0.1, momentum=0.9, scale=1.0)
    assert np.linalg.norm(_host(w) - want) <= F32 * 0.1 * np.linalg.norm(o) + 2.0 ** -23 * np.linalg.norm(want)


@pytest.mark.parametrize("cols", [1, 200, 384, 4096])
def test_singular_values_up_to_4(muon, cols):
    """A row of ones has the one singular value 1, and A is its square: 3.9 fits, 5 makes all of it NaN."""
    g = torch.ones(1, cols, device=DEV)
    inside = [(3.9, 0.0, 0.0), (1.0, -0.001, 0.0), (1.0, 0.0, 0.0)]
    assert _off(muon.orthogonalize(g, coefficients=inside), _exact(_host(g), inside)) <= F32
    assert bool(torch.isnan(muon.orthogonalize(g, coefficients=[(5.0, 0.0, 0.0), (1.0, 0.0, 0.0)])).all())


@pytest.mark.parametrize("rows,cols", [(70, 300), (300, 70), (40, 60)])
def test_singular_values_beyond_make_the_whole_matrix_nan(muon, rows, cols):
    """A, X or the polynomial does not fit: nothing of the result looks like one."""
    g = torch.zeros(rows, cols, device=DEV)
    g[3, 5] = 1.0
    for coef in ([(5.0, 0.0, 0.0), (1.0, 0.0, 0.0)], [(20.0, 0.0, 0.0), (1.0, 0.0, 0.0)]):
        got = muon.orthogonalize(g + 1e-3 * _of_norm(rows, cols, 1.0, 2), coefficients=coef)
        assert bool(torch.isnan(got).all())


@pytest.mark.parametrize("rows,cols", [(64, 96), (60, 1000), (256, 512), (512, 300)])
def test_rows_of_six_decades(muon, rows, cols):
    """A row's error: what is rounded away of X (2^-37 a number), of A (2^-37) and of the polynomial (2^-35) in each of five steps, each multiplied by at most
    3.4445 in every later one.  With at most 512 numbers in a row of the smaller side and 1000 in one of X: 1.6e-7 from X, 4e-7 from A, 1.6e-7 from the polynomial.
    The rest is relative."""
    x = torch.randn(rows, cols, generator=torch.Generator().manual_seed(5), dtype=torch.float64)
    x *= torch.logspace(0, -6, rows, dtype=torch.float64)[:, None]
    g = x.float().to(DEV)
    got, want = _host(muon.orthogonalize(g)), _exact(_host(g))
    assert np.linalg.norm(got - want) <= F32 * np.linalg.norm(want)
    assert np.all(np.linalg.norm(got - want, axis=1) <= 8e-7 + F32 * np.linalg.norm(want, axis=1))

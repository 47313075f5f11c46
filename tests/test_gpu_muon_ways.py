"""Newton-Schulz through every kind of tiles that the rule can pick (_muon_ways.py), wide and tall, against float64 products on the GPU.

Tolerances as in test_gpu_muon.py: 2e-5 of the 2-norm, a bf16 result 2^-8 more.
"""
import pytest

from _muon_ways import WAYS
from paper_1811_03617_amd import gvq  # noqa: F401  (the library itself)
from test_gpu_muon import DEFAULT, DEV, TOL

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def muon():
    from paper_1811_03617_amd import muon
    return muon


def _normal(shape, seed, by=1e-3):
    return by * torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _float64(g, eps=1e-7):
    x = g.double()
    turn = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if turn else x
    x = x / (x.norm() + eps)
    for a, b, c in DEFAULT:
        s = x @ x.t().contiguous()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if turn else x


def _off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("batch,m,n", list(WAYS))
@pytest.mark.parametrize("tall", [False, True])
def test_every_way(muon, batch, m, n, tall):
    g = _normal((batch, n, m) if tall else (batch, m, n), m).to(DEV)
    if batch == 1:
        g = g[0]
    got, low = muon.orthogonalize(g), muon.orthogonalize(g, dtype=torch.bfloat16)
    again = muon.orthogonalize(g.to(torch.bfloat16), dtype=torch.float32)
    for k in range(batch):
        at = (lambda t: t) if batch == 1 else (lambda t: t[k])
        want = _float64(at(g))
        assert _off(at(got), want) <= TOL[torch.float32]
        assert _off(at(low), want) <= TOL[torch.bfloat16]
        if k == batch - 1:
            assert _off(at(again), _float64(at(g).to(torch.bfloat16))) <= TOL[torch.float32]


@pytest.mark.parametrize("rows,cols", [s for m, n in ((96, 200), (69, 16532), (259, 21852), (1026, 3960)) for s in ((m, n), (n, m))])
@pytest.mark.parametrize("gdt,wdt", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_steps_in_place(muon, rows, cols, gdt, wdt):
    """Every tile of a last product updates the weight, in whole words and in rows that start anywhere: what lies beside it stays."""
    lr, beta, decay = 0.1, 0.9, 0.05
    scale = max(1.0, rows / cols) ** 0.5
    for at in (0, 3):
        g, m, w = _normal((rows, cols), 1).to(gdt).to(DEV), 2 * _normal((rows, cols), 2).to(DEV), _normal((rows, cols), 3, 2e-2).to(wdt).to(DEV)
        big = torch.full((rows, cols + 8), 3.0, dtype=wdt, device=DEV)
        view = big[:, at:at + cols]
        view.copy_(w)
        moved = beta * m.double() + g.double()
        o = _float64(g.double() + beta * moved)
        want = (1 - lr * decay) * w.double() - lr * scale * o
        muon.step(view, g, m, lr=lr, momentum=beta, weight_decay=decay)
        assert (m.double() - moved).norm() <= 2.0 ** -22 * moved.norm()
        tol = TOL[torch.float32] * lr * scale * o.norm() + 2.0 ** -22 * w.double().norm() + (2.0 ** -8 * want.norm() if wdt == torch.bfloat16 else 0)
        assert (view.double() - want).norm() <= tol
        view.fill_(3.0)
        assert bool((big == 3.0).all())


@pytest.mark.parametrize("batch,m,n", [(8, 260, 802), (1, 1026, 3960), (3, 1827, 2590)])
def test_same_bits_every_time(muon, batch, m, n):
    """With other matrices between, and in memory that held something else."""
    g, other = _normal((batch, m, n), 1).to(DEV), _normal((batch, m, n), 2).to(DEV)
    want = muon.orthogonalize(g)
    for _ in range(3):
        muon.orthogonalize(other)
        assert torch.equal(muon.orthogonalize(g), want)

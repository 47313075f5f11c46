"""The loss on a teacher's top logits: against its definition in float64, masked rows and entries, infinities, strides, in place,
its gradient against differences."""
import numpy as np
import pytest

import _layers_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def distill():
    from paper_1811_03617_amd import distill as module
    return module


def _case(rows, vocab, n, dtype, seed=0, spread=3.0):
    gen = torch.Generator().manual_seed(seed + 13 * rows + vocab)
    z = (spread * torch.randn(rows, vocab, generator=gen)).to(dtype)
    a = (3 * torch.randn(rows, n, generator=gen)).sort(1, descending=True).values.to(dtype)
    index = torch.randint(0, vocab, (rows, n), generator=gen)
    w = torch.rand(rows, generator=gen) + 0.5
    return z, a, index, w


def _np(x):
    return x.detach().double().cpu().numpy()


def _check(got, z, a, index, t, w, dtype):
    """Room: logits are scaled and centred in float32, which moves an exponent by half a step of its own size, |z| / t; a sum of powers adds
    some halves of steps; the loss is a sum of terms p (log p - log q) of either sign."""
    loss, grad = got
    zn, an, wn = _np(z), _np(a), _np(w)
    want_loss, want_grad = ref.distill(zn, an, index.cpu().numpy(), t, wn)
    ok = np.isfinite(zn)
    far = (np.where(ok, np.abs(zn), 0).max() + np.abs(np.where(np.isfinite(an), an, 0)).max()) / t
    e = ref.F32_HALF * (40 + 8 * far)
    assert (np.abs(_np(loss) - want_loss) <= wn * t * t * e * (1 + far) + ref.F32_HALF * np.abs(want_loss)).all()
    last = ref.BF16_HALF if dtype == BF16 else 0
    # q and the sum of p are at most 1 each; a place without entries has q alone
    q = np.zeros_like(zn)
    for r in range(len(zn)):
        s = zn[r] / t - (zn[r] / t)[ok[r]].max() if ok[r].any() else np.full(zn.shape[1], -np.inf)
        q[r] = np.exp(s) / np.exp(s).sum() if ok[r].any() else 0
    there = np.zeros_like(zn)
    i = index.cpu().numpy()
    for r in range(len(zn)):
        there[r, i[r][(i[r] >= 0) & (i[r] < zn.shape[1])]] = 1
    room = wn[:, None] * t * (q + there) * e
    assert (np.abs(_np(grad) - want_grad) <= room + last * (np.abs(want_grad) + room) + 2.0 ** -125).all()


SIZES = [(1, 1, 1), (3, 5, 2), (2, 64, 64), (5, 1000, 8), (7, 1001, 17), (2, 8193, 5), (3, 50021, 16), (1, 140000, 100), (33, 4096, 1), (300, 70, 3), (600, 9, 2),
         (1030, 9001, 4), (97, 33000, 5), (9, 1025, 300)]


@pytest.mark.parametrize("rows,vocab,n", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [1.0, 3.5])
def test_loss_and_gradient(distill, rows, vocab, n, dtype, t):
    z, a, index, w = (v.to(DEV) for v in _case(rows, vocab, n, dtype))
    got = distill.loss_and_gradient(z, a, index, temperature=t, weight=w)
    assert got[0].dtype == F32 and got[1].dtype == dtype
    _check(got, z, a, index, t, w, dtype)
    assert torch.equal(distill.loss(z, a, index, temperature=t, weight=w), got[0])
    ones = distill.loss_and_gradient(z, a, index, temperature=t)
    _check(ones, z, a, index, t, torch.ones_like(w), dtype)


def test_the_teacher_s_type_is_its_own(distill):
    z, a, index, w = (v.to(DEV) for v in _case(9, 300, 7, BF16))
    want = distill.loss_and_gradient(z, a, index, weight=w)
    got = distill.loss_and_gradient(z, a.float(), index, weight=w)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("rows,vocab", [(40, 1000), (6, 30011), (6, 66001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_and_entries_that_are_not_there(distill, rows, vocab, dtype):
    z, a, index, w = _case(rows, vocab, 12, dtype)
    index[0] = -1                              # no entries at all
    index[1, 1:] = -1                          # one
    index[2, ::2] = vocab                      # just behind the last, and far out
    index[3, 1] = 2 ** 40
    index[3, 2] = -2 ** 40
    index[4] = 7                               # one place twelve times
    index[5, 3] = index[5, 0]                  # and twice
    z[0] = float("nan")                        # of rows that are not looked at
    w[1] = 0
    z[1] = float("inf")
    a[2, 0] = float("nan")                     # of an entry that is not there
    z, a, index, w = z.to(DEV), a.to(DEV), index.to(DEV), w.to(DEV)
    got = distill.loss_and_gradient(z, a, index, temperature=2.0, weight=w)
    assert not got[0][:2].any() and not got[1][:2].any()
    z2, a2 = z.clone(), a.clone()
    z2[:2] = 0
    a2[2, 0] = 0
    _check(got, z2, a2, index, 2.0, w, dtype)
    assert torch.equal(distill.loss(z, a, index, temperature=2.0, weight=w), got[0])


@pytest.mark.parametrize("vocab", [40, 9001, 66001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_that_are_masked(distill, vocab, dtype):
    z, a, index, w = _case(8, vocab, 3, dtype)
    index[:] = torch.tensor([1, 5, 2])
    z[0, 6:] = -float("inf")                  # most of a row
    z[1, :1] = -float("inf")
    z[2, 30:] = torch.finfo(dtype).min        # the type's lowest value
    z[3] = torch.finfo(dtype).min             # everywhere: a softmax of equal numbers
    z[4] = -float("inf")                      # no softmax
    z[5, 9] = float("nan")
    z[6, 9] = float("inf")
    a[0, 1] = -float("inf")                   # an entry of probability 0
    z[7, 5] = -float("inf")                   # and one of another that the student rules out
    z, a, index, w = z.to(DEV), a.to(DEV), index.to(DEV), w.to(DEV)
    loss, grad = distill.loss_and_gradient(z, a, index, weight=w)
    assert torch.isnan(loss[4:7]).all() and torch.isnan(grad[4:7]).all()
    assert torch.isinf(loss[7]) and loss[7] > 0 and torch.isfinite(grad[7]).all()
    assert not grad[0, 6:].any() and not grad[2, 30:].any()
    rows = [0, 1, 2]
    _check((loss[rows], grad[rows]), torch.where(z[rows] < -1e30, torch.full_like(z[rows], -float("inf")), z[rows]), a[rows], index[rows], 1.0, w[rows], dtype)
    want = ref.distill(np.zeros((1, vocab)), _np(a[3:4]), index[3:4].cpu().numpy(), 1.0, _np(w[3:4]))
    assert np.allclose(_np(loss[3:4]), want[0], rtol=1e-5, atol=1e-5)
    assert np.allclose(_np(grad[3:4]), want[1], rtol=ref.BF16_HALF, atol=1e-6)


@pytest.mark.parametrize("vocab", [40, 9001, 66001])
def test_a_teacher_without_a_softmax(distill, vocab):
    z, a, index, w = _case(5, vocab, 4, F32)
    index[:] = torch.tensor([30, 2, 7, 2])
    a[0, 1] = float("inf")
    a[1] = -float("inf")
    a[2, 3] = float("nan")
    a[3, 0] = -float("inf")                   # one entry of none: as if it were not there
    z, a, index, w = z.to(DEV), a.to(DEV), index.to(DEV), w.to(DEV)
    loss, grad = distill.loss_and_gradient(z, a, index, temperature=2.0, weight=w)
    places = torch.zeros(vocab, dtype=torch.bool, device=DEV)
    places[[30, 2, 7]] = True
    assert torch.isnan(loss[:3]).all() and torch.isnan(grad[:3, places]).all() and torch.isfinite(grad[:3, ~places]).all()
    rest = slice(3, 5)
    _check((loss[rest], grad[rest]), z[rest], a[rest], index[rest], 2.0, w[rest], F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(9, 515), (3, 20001)])
def test_strides_windows_and_in_place(distill, rows, vocab, dtype):
    z, a, index, w = (v.to(DEV) for v in _case(rows, vocab, 6, dtype))
    want = distill.loss_and_gradient(z, a, index, weight=w)
    big = torch.full((rows, vocab + 7), float("nan"), dtype=dtype, device=DEV)
    big[:, 3:3 + vocab] = z
    wide = torch.full((rows, 11), -1, device=DEV)
    wide[:, 2:8] = index
    got = distill.loss_and_gradient(big[:, 3:3 + vocab], a, wide[:, 2:8], weight=w)
    assert torch.allclose(got[0], want[0], rtol=1e-5, atol=1e-6) and torch.allclose(got[1].float(), want[1].float(), rtol=1e-2, atol=1e-6)
    out = torch.full((rows, vocab + 5), 7.0, dtype=dtype, device=DEV)
    distill.loss_and_gradient(z, a, index, weight=w, out=out[:, 1:1 + vocab])
    assert torch.equal(out[:, 1:1 + vocab], want[1]) and (out[:, 0] == 7).all() and (out[:, 1 + vocab:] == 7).all()
    window = big[:, 3:3 + vocab]
    losses, same = distill.loss_and_gradient(window, a, index, weight=w, out=window)
    assert same is window and torch.equal(window, got[1]) and torch.equal(losses, got[0])
    assert torch.isnan(big[:, :3]).all() and torch.isnan(big[:, 3 + vocab:]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_in_pieces_by_windows_and_in_place(distill, dtype):
    rows, vocab = 5, 70001
    z, a, index, w = (v.to(DEV) for v in _case(rows, vocab, 6, dtype))
    index[0] = torch.tensor([0, vocab - 1, 35000, 35000, 8, 7])
    big = torch.full((rows, vocab + 7), float("nan"), dtype=dtype, device=DEV)
    big[:, 3:3 + vocab] = z
    window = big[:, 3:3 + vocab]
    for out in (None, torch.full((rows, vocab + 5), 7.0, dtype=dtype, device=DEV)[:, 1:1 + vocab], window):
        _check(distill.loss_and_gradient(window, a, index, weight=w, out=out), z, a, index, 1.0, w, dtype)
        if out is not None and out is not window:
            edges = torch.as_strided(out, (rows, vocab + 5), (vocab + 5, 1), 0)
            assert (edges[:, 0] == 7).all() and (edges[:, 1 + vocab:] == 7).all()
    assert torch.isnan(big[:, :3]).all() and torch.isnan(big[:, 3 + vocab:]).all()


@pytest.mark.parametrize("vocab", [50, 9000])
def test_the_gradient_against_differences(distill, vocab):
    z, a, index, w = _case(4, vocab, 5, F32)
    t = 2.0
    _, grad = distill.loss_and_gradient(z.to(DEV), a.to(DEV), index.to(DEV), temperature=t, weight=w.to(DEV))
    step = 1e-4
    for r, v in ((0, int(index[0, 0])), (1, int(index[1, 4])), (2, 0), (3, vocab - 1)):
        near = []
        for s in (step, -step):
            moved = _np(z)
            moved[r, v] += s
            near.append(ref.distill(moved, _np(a), index.numpy(), t, _np(w))[0][r])
        # a central difference in float64: off by a third derivative, step^2, and by rounding, 1e-16 / step
        assert abs((near[0] - near[1]) / (2 * step) - float(grad[r, v])) <= 1e-6


def test_many_entries_and_extreme_temperatures(distill):
    z, a, index, w = (v.to(DEV) for v in _case(5, 3000, 1024, F32))
    _check(distill.loss_and_gradient(z, a, index, weight=w), z, a, index, 1.0, w, F32)
    for t in (0.05, 100.0):
        _check(distill.loss_and_gradient(z, a, index, temperature=t, weight=w), z, a, index, t, w, F32)


def test_sizes_of_zero(distill):
    z, a, index, w = (v.to(DEV) for v in _case(4, 50, 3, F32))
    loss, grad = distill.loss_and_gradient(z[:0], a[:0], index[:0])
    assert loss.shape == (0,) and grad.shape == (0, 50)
    loss, grad = distill.loss_and_gradient(z, a[:, :0], index[:, :0])
    assert not loss.any() and not grad.any() and grad.shape == (4, 50)


def test_refusals(distill):
    from paper_1811_03617_amd import gvq
    z, a, index, w = (v.to(DEV) for v in _case(4, 50, 3, F32))
    for call in (lambda: distill.loss(z, a, index.int()), lambda: distill.loss(z, a[:, :2], index), lambda: distill.loss(z, a[:3], index[:3]),
                 lambda: distill.loss(z, a, index, weight=w[:3]), lambda: distill.loss(z, a, index, weight=w.double()),
                 lambda: distill.loss(z, a, index.cpu()), lambda: distill.loss(z.clone().requires_grad_(), a, index),
                 lambda: distill.loss(z, a.clone().requires_grad_(), index), lambda: distill.loss(z, a, index, weight=w.clone().requires_grad_()),
                 lambda: distill.loss_and_gradient(z, a.clone().requires_grad_(), index),
                 lambda: distill.loss(z.t(), a, index), lambda: distill.loss(z, a, index.t().contiguous().t()),
                 lambda: distill.loss_and_gradient(z, a, index, out=torch.empty(4, 49, device=DEV)),
                 lambda: distill.loss_and_gradient(z, a, index, out=torch.empty(4, 50, device=DEV, dtype=BF16))):
        with pytest.raises(ValueError):
            call()
    for t in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(gvq.GvqError):
            distill.loss(z, a, index, temperature=t)
    with pytest.raises(gvq.GvqError):
        distill.loss(z, torch.zeros(4, 1025, device=DEV), torch.zeros(4, 1025, device=DEV, dtype=torch.int64))


def test_another_stream_and_graphs(distill):
    cases = [tuple(v.to(DEV) for v in _case(rows, vocab, 9, F32)) for rows, vocab in ((40, 3000), (2, 60000), (300, 1000))]

    def all_of_it():
        return [o for z, a, index, w in cases for o in distill.loss_and_gradient(z, a, index, temperature=2.0, weight=w)]
    want = all_of_it()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = all_of_it()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, other))
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(all_of_it())
        graphs.append(g)
    for turn in range(4):
        for z, _, _, _ in cases:
            z.mul_(0.9)
        want = all_of_it()
        for g in graphs[::1 if turn % 2 else -1]:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(x, y) for x, y in zip(want, out)), turn

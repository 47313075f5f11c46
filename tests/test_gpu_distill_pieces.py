"""Few rows of many logits, which the loss takes in pieces: where that begins and ends, as many pieces as there are threads, streams and graphs.
Each case says whether it is in pieces, so that a change of the rule does not leave these kernels unrun."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_distill import DEV, F32, BF16, _case, _check, distill  # noqa: E402,F401

pytestmark = pytest.mark.gpu

SIZES = [(1, 65535, 5, False), (1, 65536, 5, True), (96, 65536, 8, True), (97, 65536, 8, False), (50, 80001, 3, True), (1, 600001, 100, True), (2, 524288, 1, True)]


def _in_pieces(rows, vocab, n):
    from paper_1811_03617_amd import gvq
    return gvq.gvq_distill_workspace(rows, vocab, n) > 0


@pytest.mark.parametrize("rows,vocab,n,pieces", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [1.0, 3.5])
def test_where_rows_are_taken_in_pieces(distill, rows, vocab, n, pieces, dtype, t):  # noqa: F811
    assert _in_pieces(rows, vocab, n) == pieces
    z, a, index, w = (v.to(DEV) for v in _case(rows, vocab, n, dtype))
    index[0, 0] = vocab - 1
    got = distill.loss_and_gradient(z, a, index, temperature=t, weight=w)
    _check(got, z, a, index, t, w, dtype)
    assert torch.equal(distill.loss(z, a, index, temperature=t, weight=w), got[0])


@pytest.mark.parametrize("t", [2.0, 20.0])
def test_pieces_on_another_stream_and_in_graphs(distill, t):  # noqa: F811
    sizes = ((2, 70001), (96, 65536), (1, 600001))
    assert all(_in_pieces(rows, vocab, 9) for rows, vocab in sizes)
    cases = [tuple(v.to(DEV) for v in _case(rows, vocab, 9, F32)) for rows, vocab in sizes]

    def all_of_it():
        return [o for z, a, index, w in cases for o in distill.loss_and_gradient(z, a, index, temperature=t, weight=w)]
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

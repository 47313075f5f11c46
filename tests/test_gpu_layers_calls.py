"""The library's own calls of the 8-bit layers, the gated block and the loss (gvq.gvq_i8_*, gvq.gvq_distill), with buffers and workspaces of the
caller's: the same bits as from the modules that make the buffers themselves."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS, N_IN, N = 70, 200, 65


def _numbers(*shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(sum(shape))).to(DEV)


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def _matrix(rows, cols):
    from paper_1811_03617_amd import gvq
    return _bytes(gvq.gvq_i8_code_bytes(rows, cols)).view(torch.int8), torch.empty(rows, device=DEV)


def test_every_call_with_the_caller_s_buffers():
    from paper_1811_03617_amd import distill, gvq, i8
    x, dy, dh, w = _numbers(ROWS, N_IN), _numbers(ROWS, 2 * N), _numbers(ROWS, N), _numbers(2 * N, N_IN)
    q, qt = i8.quantize_both(w)
    codes, codes_t = _matrix(2 * N, N_IN), _matrix(N_IN, 2 * N)
    gvq.gvq_i8_quantize(w, gvq.F32, 2 * N, N_IN, N_IN, *codes, *codes_t, _bytes(gvq.gvq_i8_quantize_workspace(2 * N, N_IN)))
    for got, want in ((codes, q), (codes_t, qt)):
        assert torch.equal(got[0], want.codes.flatten()) and torch.equal(got[1], want.scales)
    out = torch.empty(2 * N, N_IN, dtype=torch.bfloat16, device=DEV)
    gvq.gvq_i8_dequantize(*codes, 2 * N, N_IN, out, gvq.BF16, N_IN)
    assert torch.equal(out, i8.dequantize(q, torch.bfloat16))
    out = torch.ones(2 * N, 2 * N + 3, device=DEV)
    gvq.gvq_i8_matmul(*codes, *codes, 2 * N, 2 * N, N_IN, out, gvq.F32, 2 * N + 3, accumulate=True)
    assert torch.equal(out[:, :2 * N], i8.matmul(q, q, out=torch.ones(2 * N, 2 * N, device=DEV), accumulate=True)) and (out[:, 2 * N:] == 1).all()

    space = _bytes(gvq.gvq_i8_linear_workspace(ROWS, N_IN))
    y = torch.empty(ROWS, 2 * N, device=DEV)
    gvq.gvq_i8_linear(x, gvq.F32, ROWS, N_IN, N_IN, *codes, 2 * N, y, gvq.F32, 2 * N, space)
    assert torch.equal(y, i8.linear(x, q))
    h = torch.empty(ROWS, N, device=DEV)
    gvq.gvq_i8_gated(x, gvq.F32, ROWS, N_IN, N_IN, *codes, N, gvq.GELU, h, gvq.F32, N, space)
    assert torch.equal(h, i8.gated(x, q, activation="gelu"))
    gvq.gvq_i8_gated_gradient(dh, N, x, N_IN, gvq.F32, ROWS, N_IN, N, *codes, gvq.SILU, y, 2 * N, space)
    assert torch.equal(y, i8.gated_gradient(dh, x, q))

    dx, dw = torch.empty_like(x), torch.empty_like(w)
    gvq.gvq_i8_linear_backward(dy, 2 * N, x, N_IN, gvq.F32, ROWS, N_IN, 2 * N, *codes_t, dx, gvq.F32, N_IN, dw, gvq.F32, N_IN, False,
                               _bytes(gvq.gvq_i8_linear_backward_workspace(ROWS, N_IN, 2 * N)))
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), i8.linear_backward(dy, x, qt)))
    gvq.gvq_i8_gated_backward(dh, N, x, N_IN, gvq.F32, ROWS, N_IN, N, *codes, *codes_t, gvq.SILU, dx, gvq.F32, N_IN, dw, gvq.F32, N_IN, False,
                              _bytes(gvq.gvq_i8_gated_backward_workspace(ROWS, N_IN, N)))
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), i8.gated_backward(dh, x, q, qt)))

    for rows, vocab in ((9, 500), (3, 70001)):
        z, top, weight = _numbers(rows, vocab), _numbers(rows, 4), torch.rand(rows, device=DEV)
        index = torch.randint(0, vocab, (rows, 4), device=DEV)
        losses, grad = torch.empty(rows, device=DEV), torch.empty_like(z)
        gvq.gvq_distill(z, gvq.F32, rows, vocab, vocab, top, gvq.F32, index, 4, 4, 4, weight, 2.0, losses, grad, vocab,
                        _bytes(gvq.gvq_distill_workspace(rows, vocab, 4)))
        assert all(torch.equal(a, b) for a, b in zip((losses, grad), distill.loss_and_gradient(z, top, index, temperature=2.0, weight=weight)))


def test_one_gradient_in_the_workspace_that_the_header_names():
    """And not a byte behind it."""
    from paper_1811_03617_amd import gvq, i8
    x, dy, dh = _numbers(ROWS, N_IN), _numbers(ROWS, 2 * N), _numbers(ROWS, N)
    q, qt = i8.quantize_both(_numbers(2 * N, N_IN))
    one, peaks = gvq.gvq_i8_linear_workspace, gvq.gvq_i8_quantize_workspace
    for_dx = one(ROWS, 2 * N)
    for_dw = one(2 * N, ROWS) + peaks(ROWS, 2 * N) + one(N_IN, ROWS) + peaks(ROWS, N_IN)
    dg = (8 * ROWS * N + 255) // 256 * 256

    def guarded(n, run):
        space = torch.full((n + 256,), 77, dtype=torch.uint8, device=DEV)
        run(space)
        assert (space[n:] == 77).all()
    dx, dw = torch.empty(ROWS, N_IN, device=DEV), torch.empty(2 * N, N_IN, device=DEV)
    size = (gvq.F32, ROWS, N_IN)
    guarded(for_dx, lambda s: gvq.gvq_i8_linear_backward(dy, 2 * N, x, N_IN, *size, 2 * N, qt.codes, qt.scales, dx, gvq.F32, N_IN, None, gvq.F32, N_IN, False, s))
    guarded(for_dw, lambda s: gvq.gvq_i8_linear_backward(dy, 2 * N, x, N_IN, *size, 2 * N, None, None, None, gvq.F32, N_IN, dw, gvq.F32, N_IN, False, s))
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), i8.linear_backward(dy, x, qt)))
    guarded(dg + max(one(ROWS, N_IN), for_dx), lambda s: gvq.gvq_i8_gated_backward(
        dh, N, x, N_IN, *size, N, q.codes, q.scales, qt.codes, qt.scales, gvq.SILU, dx, gvq.F32, N_IN, None, gvq.F32, N_IN, False, s))
    guarded(dg + max(one(ROWS, N_IN), for_dw), lambda s: gvq.gvq_i8_gated_backward(
        dh, N, x, N_IN, *size, N, q.codes, q.scales, None, None, gvq.SILU, None, gvq.F32, N_IN, dw, gvq.F32, N_IN, False, s))
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), i8.gated_backward(dh, x, q, qt)))

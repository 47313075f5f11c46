"""The quantiser inside the products of one to four rows: every finite bf16 number beside larger ones, and fp32 numbers around every tie.

The weight is the unit matrix times a power of two, so the result is the quantised input itself, exactly; the power brings what
would be a denormal result into fp32's ordinary range.
"""
import numpy as np
import pytest

import _mx_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def mx():
    from paper_1811_03617_amd import mx
    return mx


def _through_a_layer(mx, blocks, dtype, n):
    """What blocks [N][32] become in rows of n numbers, four rows a call."""
    per = n // 32 * 4
    want = ref.quantized(blocks.astype(np.float64))
    small = np.abs(blocks).max(1) < 2.0 ** -40
    for which, up in ((small, 100), (~small, 0)):
        q = mx.quantize(2.0 ** up * torch.eye(n, device=DEV))
        some = np.flatnonzero(which)
        for at in range(0, some.size, per):
            part = some[at:at + per]
            x = np.zeros((per, 32), blocks.dtype)
            x[:part.size] = blocks[part]
            t = torch.from_numpy(x.reshape(4, n)).to(dtype).to(DEV)
            got = mx.linear(t, q, torch.float32).double().cpu().numpy().reshape(per, 32)[:part.size]
            assert np.array_equal(got, np.ldexp(want[part], up))
            one = mx.linear(t[:1], q, torch.float32)   # a row alone
            assert torch.equal(one, mx.linear(t, q, torch.float32)[:1])


def _every_bf16():
    f = (np.arange(0, 0x7F80, dtype=np.uint32) << 16).view(np.float32)
    blocks = []
    for up in (0, 1, 2, 3, 4):
        b = np.zeros((f.size, 32), np.float32)
        with np.errstate(over="ignore"):
            top = np.minimum(f * np.float32(2.0 ** up), np.float32(3.3895314e38))
        # the number and the larger one at different places of the block and of a word
        i = np.arange(f.size)
        b[i, i % 16] = f
        b[i, 16 + i % 15] = -f
        b[i, 31 - i % 2] = top
        blocks.append(b)
    return np.concatenate(blocks)


def test_every_bf16_number(mx):
    _through_a_layer(mx, _every_bf16(), torch.bfloat16, 4096)


def test_every_eleventh_bf16_number_in_a_short_sum(mx):
    _through_a_layer(mx, _every_bf16()[::11], torch.bfloat16, 96)


@pytest.mark.parametrize("n", [4096, 96])
def test_fp32_numbers_around_every_tie(mx, n):
    """At scales from the smallest to the largest: the eight magnitudes, the ties between them and their neighbours in fp32."""
    points = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7], np.float32)
    rows = []
    for e in range(-127, 126, 1 if n == 4096 else 5):
        s = np.float32(2.0 ** e) if e >= -126 else np.float32(2.0 ** -127)
        p = points * s
        b = np.zeros((3, 32), np.float32)
        b[0, :16], b[0, 16:] = p, -p
        b[1, :16], b[1, 16:] = np.nextafter(p, np.float32(np.inf)), -np.nextafter(p, np.float32(np.inf))
        b[2, :16], b[2, 16:] = np.nextafter(p, np.float32(0)), -np.nextafter(p, np.float32(0))
        b[:, 15] = 7 * s      # each block's scale is s
        rows.append(b)
    _through_a_layer(mx, np.concatenate(rows), torch.float32, n)


@pytest.mark.parametrize("rows", [1, 2, 4])
@pytest.mark.parametrize("n", [512, 100])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nan_stays_in_its_row_and_column(mx, rows, n, dtype):
    """An infinity or a NaN makes its block NaN, and with it its row of the result, of the weight its column; the others are as without it."""
    g = torch.Generator().manual_seed(n)
    x, w = torch.randn(rows, n, generator=g).to(dtype).to(DEV), torch.randn(70, n, generator=g).to(DEV)
    clean = mx.linear(x, mx.quantize(w), torch.float32)
    assert bool(torch.isfinite(clean).all())
    for value in (float("nan"), float("inf"), float("-inf")):
        for at in (0, n - 1):
            bad_x, bad_w = x.clone(), w.clone()
            bad_x[rows - 1, at] = value
            bad_w[11, at] = value
            got = mx.linear(bad_x, mx.quantize(bad_w), torch.float32)
            want = clean.clone()
            want[rows - 1] = float("nan")
            want[:, 11] = float("nan")
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))

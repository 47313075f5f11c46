"""The loss on a teacher's top logits at the ends of its ranges: entries that the student's mask covers with the type's lowest value."""
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


def _np(x):
    return x.detach().double().cpu().numpy()


@pytest.mark.parametrize("vocab", [40, 3001, 9001, 66001])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [0.5, 1.0, 4.0])
def test_entries_under_a_mask_of_the_lowest_value(distill, vocab, dtype, t):
    """Their loss is as large as the type's numbers get, and finite where its value is.  Room: p by an exponent that is rounded in float32
    (|a| / t counts) and sums of a few powers; differences of 1e38 leave nothing else."""
    gen = torch.Generator().manual_seed(vocab)
    z = torch.randn(4, vocab, generator=gen).to(dtype)
    a = torch.randn(4, 3, generator=gen).to(dtype)
    index = torch.tensor([[1, 5, 2]]).expand(4, 3).contiguous()
    w = torch.full((4,), 0.01)
    z[0, 5] = torch.finfo(dtype).min
    z[1, [5, 2]] = torch.finfo(dtype).min      # two, whose sum is no float32 number
    a[1] = 0
    z[2, 5] = torch.finfo(dtype).min           # and a difference that is none
    z[2, 30] = 3e38
    want_loss, want_grad = ref.distill(_np(z), _np(a), index.numpy(), t, _np(w))
    assert (want_loss[:3] > 1e30).all() and (want_loss < 1e38).all()
    room = ref.F32_HALF * (40 + 16 * float(a.float().abs().max()) / t)
    for out in (None, z.to(DEV)):
        loss, grad = distill.loss_and_gradient(z.to(DEV) if out is None else out, a.to(DEV), index.to(DEV), temperature=t, weight=w.to(DEV), out=out)
        assert (np.abs(_np(loss) - want_loss) <= room * (np.abs(want_loss) + 0.01 * t * t)).all()
        last = ref.BF16_HALF if dtype == BF16 else 0
        assert (np.abs(_np(grad) - want_grad) <= 0.01 * t * room + last * np.abs(want_grad)).all()
    assert torch.equal(distill.loss(z.to(DEV), a.to(DEV), index.to(DEV), temperature=t, weight=w.to(DEV)), loss) or vocab == 66001

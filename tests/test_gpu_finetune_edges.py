"""GPU: adapters and distillation where numbers end, against the definitions in 64 bits."""
import pytest
import torch

from paper_2512_02010_amd import finetune as F

from .test_gpu_distill import INF, _close, _definition, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tau", [0.1, 0.7, 1.0, 3.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1000, 40003, 131072, 270000])
def test_rows_of_the_lowest_value(V, dtype, tau):
    """A row masked by the type's lowest value throughout, or by it and -inf, is as good as one of zeros: every word the same.  Its
    lowest value divided by a temperature below 1 is no number of fp32 any more."""
    s = _inputs(4, V, 20, dtype, pad=False)
    z, low = s["logits"], torch.finfo(dtype).min
    z[0] = low
    z[1, ::2] = -INF
    z[1].scatter_(0, s["index"][1].long(), 1.0)
    z[1][z[1] > -INF] = low
    same = dict(s, logits=torch.where(z == low, 0, z))
    (loss_ref, _, d_ref), (loss_off, _, d_off) = _definition(same, tau)
    args = (z, s["teacher"], s["index"])
    loss, lse = F.nvfp4_distill_forward(*args, tau)
    step_loss, d = F.nvfp4_distill_step(*args, s["weight"], tau)
    for got, ref, off, what in ((loss, loss_ref, loss_off, "loss"), (step_loss, loss_ref, loss_off, "step's loss"), (d, d_ref, d_off, "step's dlogits")):
        _close(got, ref, off, what)
    assert bool((lse[:2] == -INF).all()) == (tau < 1)


@pytest.mark.parametrize("V", [1000, 131072, 270000])
def test_rows_of_nothing(V):
    """A row of nothing but -inf has no distribution if its list has entries, and is not learnt from if it has none."""
    s = _inputs(4, V, 20, torch.float32, pad=False)
    s["logits"][:2] = -INF
    s["index"][1] = -1
    args = (s["logits"], s["teacher"], s["index"])
    loss, lse = F.nvfp4_distill_forward(*args)
    step_loss, d = F.nvfp4_distill_step(*args, s["weight"])
    back = F.nvfp4_distill_backward(*args, lse, s["weight"])
    assert lse[:2].tolist() == [-INF, -INF]
    for t in (loss, step_loss):
        assert bool(t[0].isnan()) and float(t[1]) == 0 and bool(t[2:].isfinite().all())
    for t in (d, back):
        assert bool(t[0].isnan().all()) and not bool(t[1].any()) and bool(t[2:].isfinite().all())

"""GPU: adapters and distillation where numbers end, against the definitions in 64 bits."""
import pytest
import torch

from paper_2512_02010_amd import finetune as F

from .test_gpu_adapters import TINY, U
from .test_gpu_distill import INF, _close, _definition, _inputs
from .test_gpu_finetune_loops import _adapters

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


BITS = [(5, 1), (90, 8), (190, 16), (70, 40), (150, 100), (300, 1), (700, 12), (1000, 16), (900, 32), (800, 33), (600, 64), (700, 128)]


def _canceled(v):
    """BF16 numbers that cancel v to 2^-8 of it."""
    return (-v).bfloat16()


@pytest.mark.parametrize("T,r", BITS)
def test_bits_of_h_where_the_base_cancels(T, r):
    """Every column has one rank, and base cancels what it adds: what is left are the low bits of h, all 24 of which count, in BF16 as
    well.  Roundings: s h, three terms' sum in the matrix unit (2 u each), the addition to base, the result's own."""
    s = _adapters(T, 264, 136, r, 3, "mixed")
    columns = torch.arange(136, device="cuda")
    s["b"] = torch.where((torch.arange(r, device="cuda") == columns[:, None] % r)[None], s["b"], 0)
    _, h = F.nvfp4_adapters_forward(s["x"], None, s["a"], s["b"], s["which"], s["scales"], want_h=True)
    with_one = s["which"] >= 0
    l = s["which"].clamp(min=0).long()
    value = s["scales"].double()[l][:, None] * h.double()[:, columns % r] * s["b"].double()[l][:, columns, columns % r]
    base = torch.where(with_one[:, None], _canceled(value), s["base"])
    out = F.nvfp4_adapters_forward(s["x"], base, s["a"], s["b"], s["which"], s["scales"])
    ref = base.double() + torch.where(with_one[:, None], value, 0)
    _close(out, ref, 10 * U * value.abs() + 2.0 ** -8 * ref.abs() + TINY, "out")


@pytest.mark.parametrize("T,r", BITS)
def test_bits_of_dh_where_dx_base_cancels(T, r):
    """The same of dx; dy has one column a token, so that dh is a product, and s dh its rounding."""
    s = _adapters(T, 136, 264, r, 3, "mixed")
    columns, tokens = torch.arange(136, device="cuda"), torch.arange(T, device="cuda")
    s["a"] = torch.where((torch.arange(r, device="cuda")[:, None] == columns % r)[None], s["a"], 0)
    s["dy"] = torch.where(torch.arange(264, device="cuda") == tokens[:, None] % 264, s["dy"], 0)
    with_one = s["which"] >= 0
    l = s["which"].clamp(min=0).long()
    dh = (s["dy"].double()[tokens, tokens % 264][:, None] * s["b"].double()[l, tokens % 264])
    dh = (dh.float() * s["scales"][l][:, None]).double()
    value = dh[:, columns % r] * s["a"].double()[l][:, columns % r, columns]
    base = torch.where(with_one[:, None], _canceled(value), s["dx_base"])
    h = torch.zeros((T, r), device="cuda")
    dx = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], base)[0]
    ref = base.double() + torch.where(with_one[:, None], value, 0)
    _close(dx, ref, 10 * U * value.abs() + 2.0 ** -8 * ref.abs() + TINY, "dx")

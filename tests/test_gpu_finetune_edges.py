"""GPU: adapters and distillation where numbers end, against the definitions in 64 bits."""
import pytest
import torch

from paper_2512_02010_amd import finetune as F

from .test_gpu_adapters import TINY, U, _forward_64, _rounded, _selected
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


@pytest.mark.parametrize("value", [INF, float("nan")])
@pytest.mark.parametrize("V", [1000, 131072, 270000])
def test_rows_with_a_word_that_is_no_number(V, value):
    """All results of such a row are NaN, and nothing of the others'."""
    s = _inputs(4, V, 20, torch.float32, pad=False)
    s["logits"][1, V // 2] = value
    args = (s["logits"], s["teacher"], s["index"])
    loss, lse = F.nvfp4_distill_forward(*args)
    step_loss, d = F.nvfp4_distill_step(*args, s["weight"])
    back = F.nvfp4_distill_backward(*args, lse, s["weight"])
    for t in (loss, lse, step_loss, d, back):
        assert bool(t[1].isnan().all()) and bool(t[[0, 2, 3]].isfinite().all())


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


INFINITE = [(20, 64, 48, 8, 3, "mixed"), (150, 256, 264, 16, 4, "mixed"), (150, 264, 264, 90, 4, "mixed"), (40, 64, 72, 1, 2, "mixed"),
            (700, 264, 136, 12, 3, "segments"), (700, 264, 136, 64, 3, "mixed"), (1000, 136, 264, 128, 2, "mixed"), (1500, 264, 264, 5, 3, "mixed"),
            (9000, 264, 8192, 32, 3, "segments"), (17000, 264, 4096, 16, 3, "mixed"), (5000, 8192, 264, 33, 3, "segments"),
            (4000, 264, 8192, 60, 2, "mixed"), (3000, 4096, 264, 100, 2, "mixed")]


def _scattered(t, n, seed):
    """`t` with infinities of either sign in n places and NaN in one more."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randperm(t.numel(), generator=g)[:n + 1].to(t.device)
    t = t.clone()
    t.view(-1)[at[:n]] = torch.where(torch.arange(n, device=t.device) % 2 == 0, INF, -INF).to(t.dtype)
    t.view(-1)[at[n]] = float("nan")
    return t


def _as_defined(got, ref, close, off, what):
    """Infinities and NaN where the definition has them; elsewhere within `off` of the definition without them."""
    got = got.double()
    assert torch.equal(got.isnan(), ref.isnan()), (what, "NaN", int((got.isnan() != ref.isnan()).sum()))
    infinite = ref.isinf()
    assert torch.equal(got[infinite], ref[infinite]), (what, "infinities")
    bad = ref.isfinite() & ((got - close).abs() > off)
    assert not bool(bad.any()), (what, int(bad.sum()))


def _forward_definition(s):
    x, a, b, sc = (s[k].double() for k in ("x", "a", "b", "scales"))
    h, out = x.new_zeros((len(x), a.shape[1])), s["base"].double()
    for i, t in _selected(s):
        h[t] = _product(x[t], a[i].T)
        out[t] += sc[i] * _product(h[t], b[i].T)
    return h, out


def _product(a, b):
    """a @ b, where an element that is not finite meets whole rows and columns only (library products may pad with it)."""
    close = a.nan_to_num(0, 0, 0) @ b.nan_to_num(0, 0, 0)
    for i in (~a.isfinite()).any(1).nonzero()[:, 0].tolist():
        close[i] = (a[i][:, None] * b).sum(0)
    for j in (~b.isfinite()).any(0).nonzero()[:, 0].tolist():
        close[:, j] = (a * b[:, j]).sum(1)
    return close


@pytest.mark.parametrize("where", ["x", "a", "b", "base"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,K,N,r,adapters,order", INFINITE)
def test_infinities_forward(T, K, N, r, adapters, order, dtype, where):
    """Infinities and NaN come out where fp32 arithmetic has them, with its signs, whatever h is split into."""
    s = _adapters(T, K, N, r, adapters, order, dtype)
    s[where] = _scattered(s[where], 4, 7)
    out, h = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True)
    h_ref, ref = _forward_definition(s)
    clean = {k: v.nan_to_num(0, 0, 0) if v.is_floating_point() else v for k, v in s.items()}
    h_close, h_off, close, off = _forward_64(clean, clean["base"], 2 if dtype == torch.bfloat16 else 3)
    _as_defined(h, h_ref, h_close, h_off, "h")
    _as_defined(out, ref, close, _rounded(off, close, dtype), "out")


@pytest.mark.parametrize("where", ["dy", "x", "a", "b"])
@pytest.mark.parametrize("T,K,N,r,adapters,order", INFINITE)
def test_infinities_backward(T, K, N, r, adapters, order, where):
    s = _adapters(T, K, N, r, adapters, order)
    h = _forward_64(s, None, 2)[0].float()
    s[where] = _scattered(s[where], 4, 9)
    got = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    clean = {k: v.nan_to_num(0, 0, 0) if v.is_floating_point() else v for k, v in s.items()}
    result = []
    for v in (s, clean):
        x, dy, a, b, sc = (v[k].double() for k in ("x", "dy", "a", "b", "scales"))
        dx, da, db = v["dx_base"].double(), torch.zeros_like(a), torch.zeros_like(b)
        off = [torch.zeros_like(dx), torch.zeros_like(da), torch.zeros_like(db)]
        for i, t in _selected(v):
            n = len(t)
            dh = sc[i] * _product(dy[t], b[i])
            hs = h[t].double() * sc[i]
            dx[t] += _product(dh, a[i])
            da[i], db[i] = _product(dh.T, x[t]), _product(dy[t].T, hs)
            if v is clean:
                dh_off = 2 * (N + 8) * U * sc[i] * (dy[t].abs() @ b[i].abs()) + TINY
                off[0][t] += dh_off @ a[i].abs() + (4 * (r + 16) * U + 2.0 ** -16) * (dh.abs() @ a[i].abs()) + 4 * U * dx[t].abs() + TINY
                off[1][i] = dh_off.T @ x[t].abs() + (6 * (n + 64) * U + 2.0 ** -24) * (dh.abs().T @ x[t].abs()) + TINY
                off[2][i] = (6 * (n + 64) * U + 2.0 ** -24 + 4 * U) * (dy[t].abs().T @ hs.abs()) + TINY
        result.append((dx, da, db))
    off[0] = _rounded(off[0], result[1][0], torch.bfloat16)
    for u, ref, close, o, what in zip(got, *result, off, ("dx", "da", "db")):
        _as_defined(u, ref, close, o, what)

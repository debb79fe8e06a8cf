"""GPU: distillation from a teacher's top logits against its definition in 64 bits.

Tolerances, from the arithmetic alone (u = 2^-24).  y = z / temperature, D = max y - y:
  sum of exponentials: the exponents' rounding, 4 u D each and thus 4 u E_q[D] of the sum; the additions of a lane and the joins of
                   its 64 or more, (V / 64 + 64) 2 u; the exponential itself, 8 u
  lse              that, and 4 u (|max y| + |lse|)
  p                the same of the teacher's list
  loss             lse's, p's through every term, and 8 u (|log p| + |y| + |lse|) of it
  dlogits          exp(y - lse): lse's and 8 u (|y| + |lse|) + 8 u of itself; p's; one rounding to the logits' type
"""
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import finetune as F

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 1e-36
INF = float("inf")


def _inputs(T, V, k, dtype=torch.bfloat16, seed=1, pad=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = 2.5 * torch.randn((T, V), generator=g, device="cuda")
    teacher, index = (z + 0.7 * torch.randn((T, V), generator=g, device="cuda")).topk(min(k, V), dim=1)
    if k > V:                                          # lists longer than the vocabulary: the rest repeats words
        more = torch.randint(0, V, (T, k - V), generator=g, device="cuda")
        teacher, index = torch.cat([teacher, teacher.gather(1, more) - 1], 1), torch.cat([index, index.gather(1, more)], 1)
    index = index.to(torch.int32)
    if pad and T > 1:
        length = torch.randint(0, k + 1, (T, 1), generator=g, device="cuda")
        length[0], length[1] = k, 0
        index[torch.arange(k, device="cuda")[None] >= length] = -1
    return dict(logits=z.to(dtype), teacher=teacher.contiguous(), index=index.contiguous(),
                weight=torch.randn(T, generator=g, device="cuda"))


def _definition(s, tau, lse=None):
    """(loss, lse, dlogits) and how far each may be off."""
    z, t, at = s["logits"].double(), s["teacher"].double() / tau, s["index"].long()
    V, k = z.shape[1], at.shape[1]
    valid = (at >= 0) & (at < V) & (t > -INF)
    at = torch.where(valid, at, 0)
    y = z / tau
    m = y.amax(1)
    e = (y - m[:, None]).exp()
    depth = torch.where(e > 0, e * (m[:, None] - y), 0).sum(1) / e.sum(1)
    lse_off = 4 * U * depth + (V / 64 + 64) * 2 * U + 8 * U
    ref = m + e.sum(1).log()
    lse_off = lse_off + 4 * U * (m.abs() + ref.abs())
    if lse is not None:
        ref, lse_off = lse.double(), torch.zeros_like(lse_off)
    any_ = valid.any(1)
    log_p = torch.log_softmax(t.masked_fill(~valid, -1e300), 1)
    p = torch.where(valid, log_p.exp(), 0)
    tm = torch.where(any_, t.masked_fill(~valid, -INF).amax(1), 0)
    deep = torch.where(valid, p * (tm[:, None] - t), 0).sum(1)
    p_rel = 4 * U * (torch.where(valid, tm[:, None] - t, 0) + deep[:, None]) + (k / 64 + 64) * 2 * U + 16 * U
    yi = y.gather(1, at)
    counted = valid & (p > 0)
    terms = torch.where(counted, p * (log_p - (yi - ref[:, None])), 0)
    loss = terms.sum(1)
    size = log_p.abs() + yi.abs() + ref.abs()[:, None]
    loss_off = any_ * lse_off + torch.where(counted, terms.abs() * p_rel + p * (p_rel + 8 * U * size), 0).sum(1) + \
        (k / 64 + 64) * 2 * U * terms.abs().sum(1) + TINY
    w = torch.ones_like(m) if s.get("weight") is None else s["weight"].double()
    g = (w / tau * any_)[:, None]
    q = (y - ref[:, None]).exp()
    d = q.clone()
    d_off = q * (lse_off[:, None] + 8 * U * (torch.where(y > -INF, y, 0).abs() + ref.abs()[:, None]) + 16 * U)
    rows = torch.arange(len(z), device=z.device)[:, None].expand(-1, k)
    d.index_put_((rows[valid], at[valid]), -p[valid], accumulate=True)
    d_off.index_put_((rows[valid], at[valid]), (p * (p_rel + k * 2 * U))[valid], accumulate=True)
    d = torch.where(any_[:, None], g * d, 0)
    half = 2.0 ** -8 if s["logits"].dtype == torch.bfloat16 else U
    d_off = torch.where(any_[:, None], g.abs() * d_off * (1 + half) + (half + 4 * U) * d.abs(), 0) + TINY
    return (loss, ref, d), (loss_off, lse_off, d_off)


def _close(got, ref, off, what):
    got = got.double()
    same = (got == ref) | (got.isnan() & ref.isnan())
    bad = ~(same | ((got - ref).abs() <= off))
    assert not bool(bad.any()), (what, int(bad.sum()), float((got - ref).abs()[bad].max()), bad.nonzero()[:4].tolist())


def _check(s, tau=1.0):
    args = (s["logits"], s["teacher"], s["index"])
    loss, lse = F.nvfp4_distill_forward(*args, tau)
    (loss_ref, lse_ref, d_ref), (loss_off, lse_off, d_off) = _definition(s, tau)
    _close(lse, lse_ref, lse_off, "lse")
    _close(loss, loss_ref, loss_off, "loss")
    step_loss, step_d = F.nvfp4_distill_step(*args, s.get("weight"), tau)
    _close(step_loss, loss_ref, loss_off, "step's loss")
    _close(step_d, d_ref, d_off, "step's dlogits")
    d = F.nvfp4_distill_backward(*args, lse, s.get("weight"), tau)
    (_, _, d_ref), (_, _, d_off) = _definition(s, tau, lse)
    _close(d, d_ref, d_off, "dlogits")
    for t in (d, step_d):
        assert t.dtype == s["logits"].dtype and t.shape == s["logits"].shape
    return loss, lse, d, step_loss, step_d


SIZES = [(1, 1, 1), (1, 7, 3), (3, 8, 8), (5, 9, 12), (2, 1000, 1), (7, 32000, 16), (33, 4099, 64), (300, 1001, 100), (20, 50021, 1024),
         (1, 65536, 7), (9, 65535, 33), (4, 131072, 64), (3, 131080, 65), (2, 200003, 256), (2, 300001, 5), (1500, 515, 20)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V,k", SIZES)
def test_against_the_definition(T, V, k, dtype):
    _check(_inputs(T, V, k, dtype), tau=1.0 if V % 2 else 2.0)


@pytest.mark.parametrize("tau", [0.1, 0.7, 1.0, 5.0, 100.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_temperatures(tau, dtype):
    _check(_inputs(40, 2003, 30, dtype), tau)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_types_of_the_list(dtype):
    s = _inputs(30, 3001, 40, dtype)
    wide = dict(s, index=s["index"].long())
    first, again = _check(s), _check(wide)
    for u, v in zip(first, again):
        assert torch.equal(u, v)
    _check(dict(s, teacher=s["teacher"].bfloat16()))
    _check(dict(wide, teacher=s["teacher"].bfloat16(), weight=None))


def test_lists_with_the_same_word_twice():
    """Entries with the same index add up, two of them or all."""
    s = _inputs(16, 700, 48, torch.float32, pad=False)
    s["index"][:8, 1::2] = s["index"][:8, ::2]
    s["index"][8:] = s["index"][8:, :1]
    s["index"][12:, 30:] = -1
    _check(s)
    _check(dict(s, logits=s["logits"].bfloat16()))


def test_entries_that_are_none():
    """Indices outside the vocabulary of either sign and teacher logits of -inf; a row of nothing else is not learnt from, whatever
    it holds."""
    s = _inputs(8, 333, 12, torch.float32, pad=False)
    s["index"][0, 3:] = 333
    s["index"][1, ::2] = -(2 ** 31)
    s["index"][2, 1:] = 2 ** 31 - 1
    s["teacher"][3, 2:9] = -INF
    s["index"][4] = -1
    s["teacher"][5] = -INF
    s["logits"][4, 5], s["logits"][5, 300] = float("nan"), INF
    args = (s["logits"], s["teacher"], s["index"])
    loss, lse = F.nvfp4_distill_forward(*args)
    for t in (F.nvfp4_distill_backward(*args, lse, s["weight"]), F.nvfp4_distill_step(*args, s["weight"])[1]):
        assert not bool(t[4:6].any())
    assert loss[4:6].tolist() == [0, 0] and F.nvfp4_distill_step(*args)[0][4:6].tolist() == [0, 0]
    s["logits"][4, 5], s["logits"][5, 300] = 0.0, 1.0
    _check(s)
    wide = dict(s, index=s["index"].long())
    wide["index"][0, 3:] = 2 ** 40
    wide["index"][1, ::2] = -(2 ** 60)
    wide["index"][2, 1:] = 2 ** 32                       # (0 if it were cut to 32 bits)
    for u, v in zip(_check(s), _check(wide)):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [1000, 40003, 131072, 270000])
def test_masked_words(V, dtype):
    """Words masked by -inf or by the type's lowest value; whole stretches of a row; a masked word in the list."""
    s = _inputs(8, V, 20, dtype, pad=False)
    z = s["logits"]
    low = torch.finfo(dtype).min
    listed = torch.zeros((8, V), dtype=torch.bool, device="cuda").scatter_(1, s["index"].long(), True)
    half = (torch.arange(V, device="cuda") < V // 2)[None]
    for row, mask in ((0, half), (1, ~half), (2, torch.rand((1, V), device="cuda") < 0.9)):
        z[row][(mask & ~listed[row:row + 1])[0]] = -INF
    for row, mask in ((3, half), (4, ~half), (5, torch.rand((1, V), device="cuda") < 0.9)):
        z[row][(mask & ~listed[row:row + 1])[0]] = low
    z[6] = low                                            # nothing but the lowest value: as good as any constant
    loss, lse, d, step_loss, step_d = _check(s)
    for t in (d, step_d):
        assert not bool(t[0][(half & ~listed[:1])[0]].any()) and bool(t.isfinite().all())
    z[6] = 1.0
    z[7, int(s["index"][7, 0])] = -INF
    args = (s["logits"], s["teacher"], s["index"])
    for got in (F.nvfp4_distill_forward(*args)[0], F.nvfp4_distill_step(*args)[0]):
        assert float(got[7]) == INF and bool(got[:7].isfinite().all())
    for t in (F.nvfp4_distill_step(*args)[1], F.nvfp4_distill_backward(*args, F.nvfp4_distill_forward(*args)[1])):
        assert bool(t.isfinite().all())


def test_nan_stays_in_its_row():
    s = _inputs(6, 2500, 10, torch.float32, pad=False)
    args = (s["logits"], s["teacher"], s["index"])
    clean = _check(s)
    s["logits"][2, 1234] = float("nan")
    loss, lse = F.nvfp4_distill_forward(*args)
    d = F.nvfp4_distill_backward(*args, lse, s["weight"])
    step_loss, step_d = F.nvfp4_distill_step(*args, s["weight"])
    others = torch.arange(6, device="cuda") != 2
    for got, was in zip((loss, lse, d, step_loss, step_d), clean):
        assert torch.equal(got[others], was[others]) and bool(got[2].isnan().all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [515, 33000, 131071])
def test_rows_that_begin_anywhere(V, dtype):
    """A stride that is no multiple of a piece, a first row that begins inside one; in place."""
    s = _inputs(9, V, 17, dtype)
    want = _check(s)
    for first, pad in ((0, 1), (0, 8), (1, 0), (3, 5), (5, 11)):
        wide = torch.full((9, V + first + pad), 3.0, dtype=dtype, device="cuda")
        view = wide[:, first:first + V]
        view.copy_(s["logits"])
        moved = dict(s, logits=view)
        got = _check(moved)
        _, _, d, _, step_d = got
        assert d.stride() == view.stride() or d.shape[0] == 1
        lse = got[1]
        out = F.nvfp4_distill_backward(view, s["teacher"], s["index"], lse, s["weight"], out=view)
        assert out.data_ptr() == view.data_ptr() and torch.equal(out, d)
        view.copy_(s["logits"])
        loss, out = F.nvfp4_distill_step(view, s["teacher"], s["index"], s["weight"], out=view)
        assert torch.equal(out, step_d) and torch.equal(loss, got[3])
        assert bool((wide[:, :first] == 3).all()) and bool((wide[:, first + V:] == 3).all())
    del want


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_offsets_past_32_bits(dtype):
    """Rows so far apart that elements, and then bytes, are no 32-bit numbers any more."""
    s = _inputs(4, 5003, 20, dtype)
    want = _check(s)
    ld = (1 << 32) // 3 + 11
    room = torch.empty(3 * ld + 5003, dtype=dtype, device="cuda")
    far = room.as_strided((4, 5003), (ld, 1))
    far.copy_(s["logits"])
    loss, lse = F.nvfp4_distill_forward(far, s["teacher"], s["index"])
    for got, was in ((loss, want[0]), (lse, want[1])):
        assert bool(((got - was).abs() <= 2.0 ** -17 * (1 + was.abs())).all())                # (rows begin elsewhere: other sums)
    d = F.nvfp4_distill_backward(far, s["teacher"], s["index"], lse, s["weight"], out=far)
    assert bool(((d - want[2]).abs() <= 2.0 ** -7 * want[2].abs() + 1e-30).all())
    far.copy_(s["logits"])
    loss, d = F.nvfp4_distill_step(far, s["teacher"], s["index"], s["weight"], out=far)
    assert bool(((loss - want[3]).abs() <= 2.0 ** -17 * (1 + want[3].abs())).all())
    assert bool(((d - want[4]).abs() <= 2.0 ** -7 * want[4].abs() + 1e-30).all())


def test_no_rows():
    s = {k: v[:0] for k, v in _inputs(4, 100, 5).items()}
    loss, lse = F.nvfp4_distill_forward(s["logits"], s["teacher"], s["index"])
    d = F.nvfp4_distill_backward(s["logits"], s["teacher"], s["index"], lse, s["weight"])
    assert loss.shape == lse.shape == (0,) and d.shape == (0, 100)
    assert F.nvfp4_distill_step(s["logits"], s["teacher"], s["index"])[1].shape == (0, 100)


def test_gradient_against_differences():
    """Central differences of the 64-bit loss along random directions."""
    s = _inputs(12, 600, 25, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(8)
    tau, eps = 1.5, 2.0 ** -12
    _, d = F.nvfp4_distill_step(s["logits"], s["teacher"], s["index"], s["weight"], tau)
    for _ in range(3):
        v = torch.randn(s["logits"].shape, generator=g, device="cuda", dtype=torch.float64)
        values = [(_definition(dict(s, logits=s["logits"].double() + e * v), tau)[0][0] * s["weight"]).sum() for e in (eps, -eps)]
        numeric = float((values[0] - values[1]) / (2 * eps))
        # the third derivative of a row is at most 2 max|v / tau|^3; d is within 2^-18 of itself
        third = float((s["weight"].double().abs() * (v.abs().amax(1) / tau) ** 3).sum()) * 2 * eps ** 2 / 6
        assert abs(numeric - float((d.double() * v).sum())) < third + 2.0 ** -18 * float((d.double() * v).abs().sum()) + 1e-9


def test_the_same_bits_again_and_from_a_graph():
    for T, V in ((3, 50021), (400, 4096), (600, 131072)):
        s = _inputs(T, V, 64)
        args = (s["logits"], s["teacher"], s["index"])
        lse = F.nvfp4_distill_forward(*args)[1]
        run = lambda: (*F.nvfp4_distill_forward(*args), F.nvfp4_distill_backward(*args, lse, s["weight"]),  # noqa: E731
                       *F.nvfp4_distill_step(*args, s["weight"]))
        want = run()
        saved, B.OUTPUT_ALLOCATOR = B.OUTPUT_ALLOCATOR, B._device_empty
        try:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got = run()
            for _ in range(3):
                for t in got:
                    t.zero_()
                graph.replay()
                torch.cuda.synchronize()
                for u, v in zip(got, want):
                    assert torch.equal(u, v)
        finally:
            B.OUTPUT_ALLOCATOR = saved


def test_on_another_stream():
    s = _inputs(200, 5000, 30)
    args = (s["logits"], s["teacher"], s["index"])
    want = F.nvfp4_distill_step(*args, s["weight"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = F.nvfp4_distill_step(*args, s["weight"], stream=side)
    loss, lse = F.nvfp4_distill_forward(*args, stream=side)
    d = F.nvfp4_distill_backward(*args, lse, s["weight"], stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(F.nvfp4_distill_forward(*args)[0], loss) and torch.equal(F.nvfp4_distill_backward(*args, lse, s["weight"]), d)


def test_refusals_of_device_tensors():
    s = _inputs(6, 100, 5)
    args = (s["logits"], s["teacher"], s["index"])
    for i, t in ((0, s["logits"].half()), (0, s["logits"][0]), (0, s["logits"].T), (1, s["teacher"][:3]), (1, s["teacher"].double()),
                 (2, s["index"].short()), (2, s["index"][:, :3]), (2, s["index"].T.contiguous().T)):
        bad = args[:i] + (t,) + args[i + 1:]
        for call in (F.nvfp4_distill_forward, F.nvfp4_distill_step, lambda *a: F.nvfp4_distill_backward(*a, s["weight"])):
            with pytest.raises(AssertionError):
                call(*bad)
    with pytest.raises(AssertionError):
        F.nvfp4_distill_backward(*args, s["weight"][:3])
    with pytest.raises(AssertionError):
        F.nvfp4_distill_step(*args, out=torch.empty((6, 104), dtype=torch.bfloat16, device="cuda")[:, :100])
    for bad, status in ((dict(temperature=0.0), 4), (dict(temperature=float("nan")), 4)):
        with pytest.raises(B.Nvfp4Error) as e:
            F.nvfp4_distill_forward(*args, **bad)
        assert e.value.status == status

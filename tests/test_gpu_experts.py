"""GPU: tokens to their experts and back against plain definitions.  Places are whole numbers and have to be equal; copies have to be equal bit for bit;
sums of n fp32 products of BF16 or fp32 numbers are within (n + 1) u of the sum of magnitudes (u = 2^-24; each product and each addition
rounds once), then comes the rounding to the output's type, half a step."""
import numpy as np
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import experts as X

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def half(dtype):
    return 2.0 ** -8 if dtype == BF16 else U


def ids_of(T, k, E, kind="uneven", seed=1, dtype=torch.int32):
    r = np.random.default_rng(seed)
    if kind == "uneven":
        p = r.random(E) ** 3 + 1e-3
        ids = r.choice(E, (T, k), p=p / p.sum())
        ids[r.random((T, k)) < 0.15] = -1
    elif kind == "one":
        ids = np.full((T, k), E - 1)
    elif kind == "none":
        ids = np.full((T, k), -1)
    elif kind == "turn":
        ids = np.arange(T * k).reshape(T, k) % E
    else:                                                   # all that means "none" among some that do not
        ids = r.choice([-1, E, 0, E - 1, 2 ** 31 - 1, -2 ** 31], (T, k))
        if dtype == torch.int64:
            ids = np.where(ids == E, E + 2 ** 32, ids)      # (0 .. E - 1 in its lower half)
    return torch.from_numpy(ids).to(dtype).cuda()


def sorted_plainly(ids, E):
    flat = ids.flatten().tolist()
    k = ids.shape[1]
    key = [i if 0 <= i < E else E for i in flat]
    order = sorted(range(len(key)), key=lambda i: key[i])
    place, token, begin = [0] * len(key), [0] * len(key), [0] * (E + 1)
    for slot, pair in enumerate(order):
        place[pair] = slot if key[pair] < E else -1 - slot
        token[slot] = pair // k if key[pair] < E else -1
    for e in range(E + 1):
        begin[e] = sum(1 for i in key if i < e) if len(key) < 2000 else int((np.array(key) < e).sum())
    return place, token, begin


@pytest.mark.parametrize("T, k, E, kind", [
    (0, 2, 4, "none"), (1, 1, 1, "one"), (1, 64, 3, "uneven"), (5, 2, 4, "none"), (63, 1, 7, "uneven"), (64, 4, 64, "uneven"),
    (300, 3, 1024, "uneven"), (1024, 4, 16, "strange"), (1025, 4, 16, "uneven"), (4097, 1, 1, "one"), (2049, 2, 130, "uneven"),
    (5000, 8, 128, "uneven"), (30000, 5, 64, "turn"), (33000, 4, 1024, "uneven"), (70000, 4, 9, "strange"), (50000, 6, 255, "none"),
])
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_sort(T, k, E, kind, dtype):
    ids = ids_of(T, k, E, kind, dtype=dtype)
    place, token, begin = X.nvfp4_experts_sort(ids, E)
    want = sorted_plainly(ids.cpu(), E)
    assert place.shape == (T, k) and token.shape == (T * k,) and begin.shape == (E + 1,)
    assert place.flatten().tolist() == want[0] and token.tolist() == want[1] and begin.tolist() == want[2]


def test_sort_with_a_lent_workspace():
    w = X.experts_workspace(20000, 4, 77)
    for T in (20000, 100, 20000):
        w.random_()
        ids = ids_of(T, 4, 77, seed=T)
        for a, b in zip(X.nvfp4_experts_sort(ids, 77, workspace=w), X.nvfp4_experts_sort(ids, 77)):
            assert torch.equal(a, b)


def slots_of(T, k, W, dtype, seed=4):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((T * k, W), generator=g).to(dtype).cuda()


ROWS = [  # T, k, W
    (0, 2, 8), (1, 1, 8), (1, 3, 4096), (2, 64, 24), (5, 2, 16), (33, 4, 56), (64, 4, 4096), (100, 6, 520), (257, 8, 2880), (1000, 2, 1032),
    (3, 5, 20000), (4100, 1, 64), (7, 2, 8192), (9, 4, 8200), (300, 9, 264), (2100, 1, 2056),
]
# rows that are written and read past the caches: 96 MB and 192 MB of slots at least, in BF16
ROWS_LARGE = [(9000, 3, 4104)]


@pytest.mark.parametrize("dtype, slot_dtype", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("T, k, W", ROWS + ROWS_LARGE)
def test_spread(T, k, W, dtype, slot_dtype):
    ids = ids_of(T, k, 6)
    place, token, begin = X.nvfp4_experts_sort(ids, 6)
    x = slots_of(T, 1, W, dtype)
    xs = X.nvfp4_experts_spread(x, place, out_dtype=int(slot_dtype == F32))
    want = torch.where((token >= 0)[:, None], x[token.clamp(min=0).long()] if T else x.new_zeros((0, W)), 0).to(slot_dtype)
    assert xs.dtype == slot_dtype and torch.equal(xs, want)


def combined(ys, place, weights, base):
    """(sum, sum of magnitudes) in 64 bits"""
    there = place >= 0
    slot = torch.where(there, place, 0).long()
    w = (torch.ones(place.shape, device="cuda") if weights is None else weights).double() * there
    ref = torch.zeros((place.shape[0], ys.shape[1]), dtype=torch.float64, device="cuda") if base is None else base.double()
    size = ref.abs()
    for j in range(place.shape[1]):
        part = w[:, j, None] * ys[slot[:, j]].double()
        ref, size = ref + part, size + part.abs()
    return ref, size


@pytest.mark.parametrize("weighted, based", [(True, True), (False, False), (True, False)])
@pytest.mark.parametrize("dtype, slot_dtype", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("T, k, W", ROWS[1:] + ROWS_LARGE)
def test_combine(T, k, W, dtype, slot_dtype, weighted, based):
    place, _, _ = X.nvfp4_experts_sort(ids_of(T, k, 6), 6)
    ys = slots_of(T, k, W, slot_dtype)
    weights = torch.rand((T, k), device="cuda") if weighted else None
    base = slots_of(T, 1, W, dtype, 5) if based else None
    y = X.nvfp4_experts_combine(ys, place, weights, base, out_dtype=int(dtype == F32))
    assert y.dtype == dtype
    ref, size = combined(ys, place, weights, base)
    off = (k + 2) * U * size
    assert bool(((y.double() - ref).abs() <= off + half(dtype) * (ref.abs() + off) + 1e-40).all())
    if based:                                           # in place
        again = base.clone()
        X.nvfp4_experts_combine(ys, place, weights, again, out=again)
        assert torch.equal(again, y)


@pytest.mark.parametrize("dtype, slot_dtype", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("T, k, W", ROWS[1:] + ROWS_LARGE)
def test_combine_backward(T, k, W, dtype, slot_dtype):
    place, _, _ = X.nvfp4_experts_sort(ids_of(T, k, 6), 6)
    ys, dy, weights = slots_of(T, k, W, slot_dtype), slots_of(T, 1, W, dtype, 6), torch.rand((T, k), device="cuda")
    dys, dw = X.nvfp4_experts_combine_backward(dy, ys, place, weights)
    assert dys.dtype == slot_dtype and dw.dtype == F32 and dw.shape == (T, k)
    there = place >= 0
    slot = torch.where(there, place, ~place).long()
    for j in range(k):
        want = weights[:, j, None].double() * dy.double() * there[:, j, None]
        off = U * want.abs()
        assert bool(((dys[slot[:, j]].double() - want).abs() <= off + half(slot_dtype) * (want.abs() + off) + 1e-40).all())
        products = dy.double() * ys[slot[:, j]].double() * there[:, j, None]
        assert bool(((dw[:, j].double() - products.sum(1)).abs() <= (W + 1) * U * products.abs().sum(1)).all())
    again, ys2 = dys.clone(), ys.clone()
    got, dw2 = X.nvfp4_experts_combine_backward(dy, ys2, place, weights, out=ys2)           # in place
    assert got is ys2 and torch.equal(ys2, again) and torch.equal(dw2, dw)


def test_gradients_by_differences():
    """Both gradients of sum(y * g) for y = combine(spread(x)), weights included, against central differences in fp32: the function is
    linear in each argument alone, so that a difference is its slope but for rounding: an error of y, (k + 2) u |y| summed over the row, over the step."""
    T, k, W, E = 12, 3, 16, 4
    place, _, _ = X.nvfp4_experts_sort(ids_of(T, k, E, seed=9), E)
    x, g, w = slots_of(T, 1, W, F32), slots_of(T, 1, W, F32, 7), 0.5 + torch.rand((T, k), device="cuda")

    def value(x, w):
        y = X.nvfp4_experts_combine(X.nvfp4_experts_spread(x, place), place, w)
        return (y.double() * g.double()).sum().item(), ((y.double() * g.double()).abs().sum().item())

    dxs, dw = X.nvfp4_experts_combine_backward(g, X.nvfp4_experts_spread(x, place), place, w)
    dx = X.nvfp4_experts_combine(dxs, place)
    step = 0.25
    for t, c in ((0, 0), (3, 5), (11, 15), (7, 8)):
        up, down = x.clone(), x.clone()
        up[t, c] += step
        down[t, c] -= step
        (a, m), (b, _) = value(up, w), value(down, w)
        off = 4 * (k + 2) * U * (m + 1) / step
        assert abs((a - b) / (2 * step) - float(dx[t, c])) <= off
    for t, j in ((0, 0), (5, 2), (11, 1)):
        up, down = w.clone(), w.clone()
        up[t, j] += step
        down[t, j] -= step
        (a, m), (b, _) = value(x, up), value(x, down)
        assert abs((a - b) / (2 * step) - float(dw[t, j])) <= 4 * (k + 2) * U * (m + 1) / step


@pytest.mark.parametrize("T, W", [(5, 24), (300, 4104)])
def test_strides(T, W):
    k = 3
    place, token, _ = X.nvfp4_experts_sort(ids_of(T, k, 4), 4)
    x = slots_of(T, 1, W + 16, BF16)[:, 8:8 + W]
    room = torch.full((T * k, W + 8), 7.0, dtype=BF16, device="cuda")
    X.nvfp4_experts_spread(x, place, out=room[:, :W])
    assert torch.equal(room[:, :W], X.nvfp4_experts_spread(x.contiguous(), place)) and bool((room[:, W:] == 7).all())
    ys, w = room[:, :W], torch.rand((T, k), device="cuda")
    y = torch.full((T, W + 40), 7.0, dtype=BF16, device="cuda")
    X.nvfp4_experts_combine(ys, place, w, base=x, out=y[:, :W])
    assert torch.equal(y[:, :W], X.nvfp4_experts_combine(ys.contiguous(), place, w, base=x.contiguous())) and bool((y[:, W:] == 7).all())
    d = torch.full((T * k, W + 24), 7.0, dtype=BF16, device="cuda")
    _, dw = X.nvfp4_experts_combine_backward(x, ys, place, w, out=d[:, :W])
    want, dw2 = X.nvfp4_experts_combine_backward(x.contiguous(), ys.contiguous(), place, w)
    assert torch.equal(d[:, :W], want) and bool((d[:, W:] == 7).all()) and torch.equal(dw, dw2)


def test_places_that_are_no_slots():
    """Left out, whatever they hold: nothing is read or written for them."""
    T, k, W = 20, 3, 64
    place, _, _ = X.nvfp4_experts_sort(ids_of(T, k, 4, "turn"), 4)
    ys, x, w = slots_of(T, k, W, F32), slots_of(T, 1, W, F32), torch.rand((T, k), device="cuda")
    bad = place.clone()
    bad[2, 1], bad[5, 0], bad[9, 2], bad[9, 1] = T * k, 2 ** 31 - 1, -2 ** 31, -1 - T * k
    lost = bad != place
    y = X.nvfp4_experts_combine(ys, bad, w)
    assert torch.equal(y, X.nvfp4_experts_combine(ys, place, w * ~lost))
    out = torch.full((T * k, W), 7.0, device="cuda")
    X.nvfp4_experts_spread(x, bad, out=out)
    full = X.nvfp4_experts_spread(x, place)
    slots = place[lost].long()
    assert bool((out[slots] == 7).all())
    full[slots] = 7
    assert torch.equal(out, full)
    out.fill_(7)
    _, dw = X.nvfp4_experts_combine_backward(x, ys, bad, w, out=out)
    want, dw2 = X.nvfp4_experts_combine_backward(x, ys, place, w)
    assert bool((out[slots] == 7).all()) and not bool(dw[lost].any()) and torch.equal(dw[~lost], dw2[~lost])
    want[slots] = 7
    assert torch.equal(out, want)


def test_what_is_masked_does_not_reach_a_sum():
    """NaN and infinities at the slots of pairs without an expert, and weights of NaN there, change nothing."""
    T, k, W = 40, 4, 72
    place, _, begin = X.nvfp4_experts_sort(ids_of(T, k, 5), 5)
    ys, dy, w = slots_of(T, k, W, BF16), slots_of(T, 1, W, BF16, 3), torch.rand((T, k), device="cuda")
    want, back = X.nvfp4_experts_combine(ys, place, w), X.nvfp4_experts_combine_backward(dy, ys, place, w)
    ys[int(begin[-1]):] = float("nan")
    w[place < 0] = float("inf")
    assert torch.equal(X.nvfp4_experts_combine(ys, place, w), want)
    dys, dw = X.nvfp4_experts_combine_backward(dy, ys, place, w)
    assert torch.equal(dys, back[0]) and torch.equal(dw, back[1])
    # ... and what is not masked does
    ys[int(place[place >= 0][0])] = float("inf")
    assert bool(X.nvfp4_experts_combine(ys, place, None).isinf().any())


def test_replayed_from_graphs_and_on_other_streams():
    """Two captured graphs of sort, spread and combine with their gradients, replayed in turn beside eager calls on another stream."""
    for T, k, E, W in ((30, 3, 5, 64), (3000, 4, 70, 264)):
        ids, x, w = ids_of(T, k, E), slots_of(T, 1, W, BF16), torch.rand((T, k), device="cuda")

        def call(stream=None):
            place, token, begin = X.nvfp4_experts_sort(ids, E, stream=stream)
            xs = X.nvfp4_experts_spread(x, place, stream=stream)
            y = X.nvfp4_experts_combine(xs, place, w, base=x, stream=stream)
            dys, dw = X.nvfp4_experts_combine_backward(y, xs, place, w, stream=stream)
            return place, token, begin, xs, y, dys, dw

        graphs = []
        for _ in range(2):
            call()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got = call()
            graphs.append((graph, got))
        side = torch.cuda.Stream()
        for _ in range(3):
            for graph, got in graphs:
                ids.copy_(torch.roll(ids, 1, 0))
                x.copy_(torch.roll(x, 3, 0))
                side.wait_stream(torch.cuda.current_stream())
                other = call(side)
                graph.replay()
                eager = call()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(eager, got, other))


def test_outputs_that_do_not_fit_are_refused():
    place, _, _ = X.nvfp4_experts_sort(ids_of(4, 2, 3), 3)
    x, xs, w = slots_of(4, 1, 64, BF16), slots_of(4, 2, 64, BF16), torch.rand((4, 2), device="cuda")
    for call, text in (
            (lambda: X.nvfp4_experts_spread(x, place, out=xs[:7]), "out must be of a shape"),
            (lambda: X.nvfp4_experts_combine(xs, place, base=x, out=x.float()), "out must be BFloat16"),
            (lambda: X.nvfp4_experts_combine_backward(x, xs, place, w, out=xs.float()), "out must be BFloat16"),
            (lambda: X.nvfp4_experts_combine_backward(x, xs, place, w, out=xs[:, :32]), "out must be of a shape")):
        with pytest.raises(AssertionError, match=text):
            call()
    with pytest.raises(B.Nvfp4Error, match="ALIGN"):
        X.nvfp4_experts_spread(x, place, out=torch.empty((8, 68), dtype=BF16, device="cuda")[:, :64])


@pytest.mark.parametrize("T, k, E", [(1, 1, 1), (37, 3, 9), (64, 4, 64), (2000, 5, 100)])
def test_outputs_that_the_calls_allocate_themselves(T, k, E, monkeypatch):
    """As in a user's program (other tests hand in an allocator): the same values, in tensors that do not overlap and may be changed apart."""
    ids, x, w = ids_of(T, k, E), slots_of(T, 1, 72, BF16), torch.rand((T, k), device="cuda")

    def call():
        place, token, begin = X.nvfp4_experts_sort(ids, E)
        xs = X.nvfp4_experts_spread(x, place)
        y = X.nvfp4_experts_combine(xs, place, w, base=x)
        return (place, token, begin, xs, y, *X.nvfp4_experts_combine_backward(y, xs, place, w))

    want = call()
    monkeypatch.setattr(B, "OUTPUT_ALLOCATOR", B._device_empty)
    got = call()
    assert all(a.shape == b.shape and a.dtype == b.dtype and a.stride() == b.stride() and torch.equal(a, b) for a, b in zip(want, got))
    spans = sorted((t.data_ptr(), t.data_ptr() + t.nbytes) for t in got)
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and all(t.data_ptr() % 256 == 0 for t in got)
    kept = [t.clone() for t in got]
    got[1].fill_(-7)
    got[0].add_(1)
    assert torch.equal(got[2], kept[2]) and bool((got[1] == -7).all()) and torch.equal(got[0], kept[0] + 1)

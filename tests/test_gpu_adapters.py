"""GPU: low-rank adapters, forwards and backwards, against their definition in 64 bits.

Tolerances, per element, from the arithmetic alone (u = 2^-24, fp32's half unit; sums of n terms in any order are within
2 n u of the sum of magnitudes, the factor 2 for the matrix unit's truncation):
  h       K products, exact each                                             2 K u sum |x a|
  delta   the same for its r terms, h's own error through B, and h in two BF16 terms (half a unit of eight bits is 2^-8:
          2^-16 of h is left) for BF16 outputs, in three for fp32 ones (2^-24)
  out     delta's, one addition, one rounding to the output's type
  dA, dB  as delta, over the adapter's tokens
"""
import numpy as np
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import finetune as F
from paper_2512_02010_amd import linear as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 1e-30


def _which(T, adapters, order, seed, none=0.2):
    r = np.random.default_rng(seed)
    if order == "mixed":
        w = r.integers(0, adapters, T)
        w[r.random(T) < none] = -1
    elif order == "segments":
        w = np.sort(r.integers(0, adapters, T))
        w = np.where(np.isin(w, r.integers(0, adapters, 1)) & (none > 0), -1, w)
    elif order == "one":
        w = np.full(T, adapters - 1)
    elif order == "none":
        w = np.full(T, -1)
    else:                                                   # all that means "none"
        w = r.choice([-1, adapters, -2 ** 31, 2 ** 31 - 1, 0], T)
    return torch.from_numpy(w.astype(np.int32))


def _inputs(T, K, N, r, adapters, order="mixed", seed=1, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g)

    s = dict(x=(normal(T, K) * torch.exp(normal(T, 1))).bfloat16(), a=(normal(adapters, r, K) / K ** 0.5).bfloat16(),
             b=(normal(adapters, N, r) / r ** 0.5).bfloat16(), which=_which(T, adapters, order, seed),
             scales=0.25 + 2 * torch.rand(adapters, generator=g), base=normal(T, N).to(dtype),
             dy=(1e-3 * normal(T, N) * torch.exp(normal(T, 1))).bfloat16(), dx_base=(1e-3 * normal(T, K)).bfloat16())
    return {k: v.cuda() for k, v in s.items()}


def _selected(s):
    """A and B of every adapter's tokens: (adapter, its tokens)"""
    for i in range(len(s["scales"])):
        yield i, (s["which"] == i).nonzero()[:, 0]


def _forward_64(s, base, terms):
    x, a, b, sc = (s[k].double() for k in ("x", "a", "b", "scales"))
    T, K = x.shape
    r = a.shape[1]
    h, h_off = x.new_zeros((T, r)), x.new_zeros((T, r))
    out = torch.zeros((T, b.shape[1]), dtype=torch.float64, device="cuda") if base is None else base.double()
    off = torch.zeros_like(out)
    split = 2.0 ** (-16 if terms == 2 else -24)
    for i, t in _selected(s):
        h[t] = x[t] @ a[i].T
        h_off[t] = 2 * K * U * (x[t].abs() @ a[i].abs().T) + TINY
        out[t] += sc[i] * (h[t] @ b[i].T)
        off[t] += sc[i] * (h_off[t] @ b[i].abs().T + (2 * terms * (r + 16) * U + split) * (h[t].abs() @ b[i].abs().T))
    return h, h_off, out, off + 4 * U * out.abs() + TINY


def _rounded(off, ref, dtype):
    half = 2.0 ** -8 if dtype == torch.bfloat16 else U
    return off + half * (ref.abs() + off) + TINY


def _close(got, ref, off, what):
    bad = (got.double() - ref).abs() > off
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - ref).abs() / off).max()))


def _check_forward(s, dtype, base=True, **kw):
    base_t = s["base"] if base else None
    out, h = F.nvfp4_adapters_forward(s["x"], base_t, s["a"], s["b"], s["which"], s["scales"], want_h=True, **kw)
    assert out.dtype == dtype and h.dtype == torch.float32
    h_ref, h_off, ref, off = _forward_64(s, base_t, 2 if dtype == torch.bfloat16 else 3)
    _close(h, h_ref, h_off, "h")
    _close(out, ref, _rounded(off, ref, dtype), "out")
    none = (s["which"] < 0) | (s["which"] >= len(s["scales"]))
    if base:
        assert torch.equal(out[none], base_t[none])
    assert not bool(h[none].any())
    return out, h


def _check_backward(s, dx_base=True, want_dx=True, h=None, **kw):
    x, dy, a, b, sc = (s[k].double() for k in ("x", "dy", "a", "b", "scales"))
    T, K = x.shape
    N, r = b.shape[1:]
    if h is None:
        h = _forward_64(s, None, 2)[0].float()
    base = s["dx_base"] if dx_base else None
    dx, da, db = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], base, want_dx, **kw)
    ref = torch.zeros_like(x) if base is None else base.double()
    off = torch.zeros_like(x)
    for i, t in _selected(s):
        n = len(t)
        dh = sc[i] * (dy[t] @ b[i])
        dh_off = 2 * (N + 8) * U * sc[i] * (dy[t].abs() @ b[i].abs()) + TINY
        ref[t] += dh @ a[i]
        off[t] += dh_off @ a[i].abs() + (4 * (r + 16) * U + 2.0 ** -16) * (dh.abs() @ a[i].abs())
        da_ref = dh.T @ x[t]
        da_off = dh_off.T @ x[t].abs() + (6 * (n + 64) * U + 2.0 ** -24) * (dh.abs().T @ x[t].abs()) + TINY
        _close(da[i], da_ref, da_off, f"da[{i}]")
        hs = h[t].double() * sc[i]
        db_off = (6 * (n + 64) * U + 2.0 ** -24 + 4 * U) * (dy[t].abs().T @ hs.abs()) + TINY
        _close(db[i], dy[t].T @ hs, db_off, f"db[{i}]")
        if n == 0:
            assert not bool(da[i].any()) and not bool(db[i].any())
    if want_dx:
        assert dx.dtype == torch.bfloat16
        _close(dx, ref, _rounded(off + 4 * U * ref.abs() + TINY, ref, torch.bfloat16), "dx")
    else:
        assert dx is None
    return dx, da, db


SIZES = [  # T, K, N, r, adapters, order
    (1, 8, 8, 1, 1, "one"), (1, 4096, 4096, 16, 4, "mixed"), (2, 64, 40, 3, 2, "mixed"), (3, 4104, 1032, 64, 2, "mixed"),
    (15, 512, 256, 8, 3, "mixed"), (16, 512, 264, 16, 16, "mixed"), (17, 520, 2048, 32, 2, "segments"), (33, 264, 72, 128, 2, "mixed"),
    (64, 2048, 2048, 16, 32, "mixed"), (65, 136, 200, 100, 3, "segments"), (100, 1000, 8, 5, 7, "strange"), (128, 8, 1000, 12, 2, "mixed"),
    (130, 256, 256, 16, 2, "none"), (257, 768, 520, 33, 5, "mixed"), (1000, 1024, 1536, 64, 8, "segments"), (1023, 320, 328, 16, 64, "mixed"),
    (1025, 520, 264, 16, 65, "mixed"), (2049, 256, 512, 8, 3, "segments"), (3001, 96, 104, 20, 300, "mixed"), (2048, 1024, 1024, 16, 1, "one"),
    (5000, 264, 136, 4, 2048, "mixed"),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,K,N,r,adapters,order", SIZES)
def test_forward(T, K, N, r, adapters, order, dtype):
    _check_forward(_inputs(T, K, N, r, adapters, order, dtype=dtype), dtype)


@pytest.mark.parametrize("T,K,N,r,adapters,order", SIZES)
def test_backward(T, K, N, r, adapters, order):
    _check_backward(_inputs(T, K, N, r, adapters, order))


@pytest.mark.parametrize("T", [1, 40, 1500])
def test_without_a_base(T):
    s = _inputs(T, 256, 192, 16, 3)
    out, _ = _check_forward(s, torch.bfloat16, base=False)
    assert out.shape == (T, 192)
    _check_backward(s, dx_base=False)
    _check_backward(s, want_dx=False)


@pytest.mark.parametrize("T", [1, 50, 1300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_rows_and_in_place(T, dtype):
    """Slices of wider matrices (a projection that gives several outputs side by side), and out = base."""
    s = _inputs(T, 264, 136, 16, 5, dtype=dtype)
    plain, h = _check_forward(s, dtype)
    wide = {k: torch.full((T, s[k].shape[1] + 48), 7.0, dtype=s[k].dtype, device="cuda") for k in ("x", "base", "dy", "dx_base")}
    for k, w in wide.items():
        w[:, 16:16 + s[k].shape[1]] = s[k]
    view = {k: w[:, 16:16 + s[k].shape[1]] for k, w in wide.items()}
    out = F.nvfp4_adapters_forward(view["x"], view["base"], s["a"], s["b"], s["which"], s["scales"], out=view["base"])
    assert out.data_ptr() == view["base"].data_ptr() and torch.equal(out, plain)
    assert bool((wide["base"][:, :16] == 7).all()) and bool((wide["base"][:, 16 + 136:] == 7).all())
    if dtype == torch.bfloat16:
        dx, da, db = _check_backward(s, h=h)
        got = F.nvfp4_adapters_backward(view["dy"], view["x"], h, s["a"], s["b"], s["which"], s["scales"], view["dx_base"],
                                        out=view["dx_base"])
        for u, v in zip(got, (dx, da, db)):
            assert torch.equal(u, v)
        assert bool((wide["dx_base"][:, :16] == 7).all()) and bool((wide["dx_base"][:, 16 + 264:] == 7).all())


@pytest.mark.parametrize("T", [3, 700, 4000])
def test_a_tokens_result_does_not_depend_on_its_place(T):
    """Permuted tokens give permuted rows, bit for bit; and the same call gives the same bits again."""
    s = _inputs(T, 512, 256, 16, 6)
    out, h = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True)
    perm = torch.randperm(T, generator=torch.Generator().manual_seed(3)).cuda()
    moved, moved_h = F.nvfp4_adapters_forward(s["x"][perm], s["base"][perm], s["a"], s["b"], s["which"][perm], s["scales"], want_h=True)
    assert torch.equal(moved, out[perm]) and torch.equal(moved_h, h[perm])
    first = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    again = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    for u, v in zip(first, again):
        assert torch.equal(u, v)


@pytest.mark.parametrize("T", [20, 1200])
def test_infinities_and_nan_stay_with_their_tokens(T):
    """A token of no number touches its own row, its own adapter's gradients, and nothing else."""
    s = _inputs(T, 256, 128, 16, 4)
    s["which"][::3] = 2
    s["which"][5] = 1
    clean, h = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True)
    back = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    x, dy, which = s["x"].clone(), s["dy"].clone(), s["which"].clone()
    x[5, 7], dy[5, 9] = float("nan"), float("inf")
    which[8], x[8], dy[8] = -1, float("nan"), float("nan")             # no adapter: its values are not looked at
    s2 = dict(s, which=which)
    ref = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], which, s["scales"])
    out, h2 = F.nvfp4_adapters_forward(x, s["base"], s["a"], s["b"], which, s["scales"], want_h=True)
    others = torch.arange(T, device="cuda") != 5
    assert torch.equal(out[others], ref[others]) and bool(out[5].isnan().all()) and torch.equal(out[8], s["base"][8])
    assert bool(h2[5].isnan().all()) and not bool(h2[8].any())
    back = F.nvfp4_adapters_backward(s["dy"], s["x"], h2.nan_to_num(), s["a"], s["b"], which, s["scales"], s["dx_base"])
    dx, da, db = F.nvfp4_adapters_backward(dy, x, h2.nan_to_num(), s["a"], s["b"], which, s["scales"], s["dx_base"])
    assert torch.equal(dx[others], back[0][others]) and torch.equal(dx[8], s["dx_base"][8])
    for i in (0, 2, 3):
        assert torch.equal(da[i], back[1][i]) and torch.equal(db[i], back[2][i])
    assert bool(da[1].isnan().any()) and not bool(db[1][9].isfinite().all())
    del clean, s2


def test_no_tokens():
    s = _inputs(4, 64, 48, 8, 3)
    for k in ("x", "base", "which", "dy", "dx_base"):
        s[k] = s[k][:0]
    out, h = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True)
    assert out.shape == (0, 48) and h.shape == (0, 8)
    dx, da, db = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    assert dx.shape == (0, 64) and not bool(da.any()) and not bool(db.any())


def test_gradients_against_differences():
    """The directional derivative of sum(out * dy), by central differences of the 64-bit definition, at the kernels' gradients."""
    s = _inputs(300, 128, 96, 8, 3)
    g = torch.Generator(device="cuda").manual_seed(9)
    v = {k: s[k].double() for k in ("x", "a", "b")}
    dy, sc = s["dy"].double(), s["scales"].double()
    dirs = {k: torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64) for k, t in v.items()}

    def value(x, a, b):
        return sum(float((sc[i] * (x[t] @ a[i].T) @ b[i].T * dy[t]).sum()) for i, t in _selected(s))

    h = _forward_64(s, None, 2)[0].float()
    dx, da, db = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], None)
    eps = 2.0 ** -10
    for k, grad in (("x", dx), ("a", da), ("b", db)):
        hi, lo = dict(v), dict(v)
        hi[k], lo[k] = v[k] + eps * dirs[k], v[k] - eps * dirs[k]
        numeric = (value(**hi) - value(**lo)) / (2 * eps)                # (the value is linear in each of the three)
        size = float((grad.double() * dirs[k]).abs().sum())
        assert abs(numeric - float((grad.double() * dirs[k]).sum())) < (2.0 ** -8 if k == "x" else 2.0 ** -17) * size, k


def test_on_another_stream_and_with_a_lent_workspace():
    s = _inputs(1500, 512, 256, 16, 4)
    want = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True)
    back = F.nvfp4_adapters_backward(s["dy"], s["x"], want[1], s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    side = torch.cuda.Stream()
    ws = [F.adapters_workspace(1500, 512, 256, 4, 16, backward) for backward in (False, True)]
    side.wait_stream(torch.cuda.current_stream())
    for w in ((None, None), ws):
        got = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True, workspace=w[0], stream=side)
        grads = F.nvfp4_adapters_backward(s["dy"], s["x"], got[1], s["a"], s["b"], s["which"], s["scales"], s["dx_base"],
                                          workspace=w[1], stream=side)
        side.synchronize()
        for u, v in zip((*got, *grads), (*want, *back)):
            assert torch.equal(u, v)
    with pytest.raises(B.Nvfp4Error) as e:
        F.nvfp4_adapters_backward(s["dy"], s["x"], want[1], s["a"], s["b"], s["which"], s["scales"], workspace=ws[1][:-16])
    assert e.value.status == 4


def test_refusals_of_device_tensors():
    s = _inputs(16, 64, 48, 8, 2)
    args = (s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"])

    def changed(i, t):
        return args[:i] + (t,) + args[i + 1:]

    for i, t in ((0, s["x"].float()), (0, s["x"][:, :56]), (0, s["x"].T.contiguous().T), (1, s["base"][:8]), (1, s["base"].half()),
                 (2, s["a"][0]), (2, s["a"].float()), (3, s["b"].transpose(1, 2)), (4, s["which"].long()), (4, s["which"][:8]),
                 (5, s["scales"].double()), (5, s["scales"][:1])):
        with pytest.raises(AssertionError):
            F.nvfp4_adapters_forward(*changed(i, t))
    for bad, status in ((dict(out=torch.empty(16 * 48 + 8, dtype=torch.bfloat16, device="cuda")[4:772].view(16, 48)), 3),):
        with pytest.raises(B.Nvfp4Error) as e:
            F.nvfp4_adapters_forward(*args, **bad)
        assert e.value.status == status


@pytest.mark.parametrize("T", [5, 300])
def test_offsets_past_32_bits(T):
    """Rows so far apart that elements, and then bytes, are no 32-bit numbers any more."""
    s = _inputs(T, 64, 48, 8, 3)
    want = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True)
    back = F.nvfp4_adapters_backward(s["dy"], s["x"], want[1], s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
    ld = ((1 << 32) // (T - 1) + 8) // 8 * 8
    room = torch.empty((T - 1) * ld + 256, dtype=torch.bfloat16, device="cuda")
    far = {k: room.as_strided((T, s[k].shape[1]), (ld, 1), at) for k, at in (("x", 0), ("base", 64), ("dy", 128), ("dx_base", 192))}
    for k, v in far.items():
        v.copy_(s[k])
    out, h = F.nvfp4_adapters_forward(far["x"], far["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True, out=far["base"])
    assert torch.equal(out, want[0]) and torch.equal(h, want[1])
    got = F.nvfp4_adapters_backward(far["dy"], far["x"], h, s["a"], s["b"], s["which"], s["scales"], far["dx_base"], out=far["dx_base"])
    for u, v in zip(got, back):
        assert torch.equal(u, v)


def test_replayed_from_a_graph():
    """Captured once and replayed: nothing is asked of the host, and nothing is left from one replay to the next."""
    s = _inputs(1100, 256, 512, 16, 3)
    run = lambda: (*F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=True),  # noqa: E731
                   )
    want = run()
    back = lambda h: F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], s["dx_base"])  # noqa: E731
    want = want + back(want[1])
    saved, B.OUTPUT_ALLOCATOR = B.OUTPUT_ALLOCATOR, B._device_empty
    try:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
            got = got + back(got[1])
        for _ in range(3):
            for t in got:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for u, v in zip(got, want):
                assert torch.equal(u, v)
    finally:
        B.OUTPUT_ALLOCATOR = saved


def test_beside_a_quantized_projection():
    """The layer of linear.py with adapters added to it is the layer, then the adapters, bit for bit."""
    g = torch.Generator(device="cuda").manual_seed(4)
    T, K, N = 96, 256, 192
    s = _inputs(T, K, N, 16, 3)
    qw = L.quantize_weight(torch.randn((N, K), generator=g, device="cuda") / 16)
    y = L.fprop(s["x"], qw)
    want, h = F.nvfp4_adapters_forward(s["x"], y, s["a"], s["b"], s["which"], s["scales"], want_h=True)
    got, h2 = F.adapted_fprop(s["x"], qw, s["a"], s["b"], s["which"], s["scales"], want_h=True)
    assert torch.equal(got, want) and torch.equal(h, h2)
    dx = L.dgrad(s["dy"], qw, 77)
    want = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], dx)
    got = F.adapted_backward(s["dy"], s["x"], h, qw, s["a"], s["b"], s["which"], s["scales"], 77)
    for u, v in zip(got, want):
        assert torch.equal(u, v)

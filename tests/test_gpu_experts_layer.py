"""GPU: a layer of experts as it is used -- sort, products, combine, and all of it backwards -- against its definition in 64 bits, step by step
from what the step before left (each step's own bound is that of its own tests: sums of n products 2 n u, u = 2^-24, and half a step of BF16, 2^-8)."""
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import experts as X
from paper_2512_02010_amd import finetune as F

from .test_gpu_experts import ids_of
from .test_gpu_weight_product import U, close, values

pytestmark = pytest.mark.gpu


def _layer(E, K, H, block2d, seed=1):
    g = torch.Generator().manual_seed(seed)
    make = lambda n, k: X.quantize_experts((torch.randn((E, n, k), generator=g) / k ** 0.5).cuda(), block2d=block2d)   # noqa: E731
    return make(H, K), make(K, H)


def _weights(q, back=False):
    """[E][N][K] in 64 bits, of the packing that the call reads"""
    c, s = (q["codes_col"], q["scales_col"]) if back else (q["codes_row"], q["scales_row"])
    w = torch.stack([q["alpha"][e].double() * values(c[e], s[e], q["block2d"]) for e in range(q["shape"][0])])
    return w.transpose(1, 2) if back else w


@pytest.mark.parametrize("T, k, E, K, H, block2d", [(1, 2, 4, 64, 96, True), (20, 3, 8, 128, 160, True), (77, 2, 5, 256, 96, False), (900, 4, 6, 256, 512, True),
                                                    (2500, 2, 16, 512, 256, False)])
def test_feed_forward_and_its_gradients(T, k, E, K, H, block2d):
    up, down = _layer(E, K, H, block2d)
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn((T, K), generator=g).bfloat16().cuda() for _ in range(2))
    ids, weights = ids_of(T, k, E), torch.rand((T, k), generator=g).cuda()
    y, kept = X.feed_forward(x, ids, weights, up, down, base=x)
    place, begin, h, ys = kept
    b = begin.tolist()
    token = torch.zeros(T * k, dtype=torch.int64, device="cuda")
    pairs = torch.arange(T, device="cuda")[:, None].expand(T, k)
    there = place >= 0
    token[place[there].long()] = pairs[there]

    def step(got, source, w, n, e):
        ref = source.double() @ w[e].T
        off = 2 * (n + 64) * U * (source.double().abs() @ w[e].abs().T) + 2 * U * ref.abs()
        close(got[b[e]:b[e + 1]], ref, off + 2.0 ** -8 * (ref.abs() + off) + 1e-30, e)

    wu, wd = _weights(up), _weights(down)
    for e in range(E):
        step(h, x[token[b[e]:b[e + 1]]], wu, K, e)
        step(ys, torch.relu(h[b[e]:b[e + 1]]), wd, H, e)
    ref, size = x.double(), x.double().abs()
    for j in range(k):
        part = (weights[:, j] * there[:, j])[:, None].double() * ys[place[:, j].clamp(min=0).long()].double()
        ref, size = ref + part, size + part.abs()
    off = (k + 2) * U * size
    close(y, ref, off + 2.0 ** -8 * (ref.abs() + off) + 1e-30, "y")

    # the gradients: of the layer with the values that the products left, h and ys, which the backward pass has too
    dx, dw = X.feed_forward_backward(dy, kept, weights, up, down)
    for j in range(k):
        products = dy.double() * ys[place[:, j].clamp(min=0).long()].double() * there[:, j, None]
        assert bool(((dw[:, j].double() - products.sum(1)).abs() <= (K + 1) * U * products.abs().sum(1)).all())
    ud, uu = _weights(down, True), _weights(up, True)
    ref, off = torch.zeros((T, K), dtype=torch.float64, device="cuda"), torch.zeros((T, K), dtype=torch.float64, device="cuda")
    half = 2.0 ** -8
    for j in range(k):
        mine = there[:, j].nonzero()[:, 0]
        slot = place[mine, j].long()
        e_of = ids[mine, j].long()
        for e in e_of.unique().tolist():
            sel = e_of == e
            t, s = mine[sel], slot[sel]
            dys = weights[t, j, None].double() * dy[t].double()
            d_off = (half + U) * dys.abs()
            dh = (dys @ ud[e]) * (h[s] > 0)
            h_off = d_off @ ud[e].abs() + 2 * (K + 64) * U * (dys.abs() @ ud[e].abs())
            h_off = (h_off + half * (dh.abs() + h_off)) * (h[s] > 0)
            dxs = dh @ uu[e]
            x_off = h_off @ uu[e].abs() + 2 * (H + 64) * U * ((dh.abs() + h_off) @ uu[e].abs())
            ref[t] += dxs
            off[t] += x_off + half * (dxs.abs() + x_off) + (k + 1) * U * (dxs.abs() + x_off)
    close(dx, ref, off + half * (ref.abs() + off) + 1e-30, "dx")


def test_adapters_beside_the_experts():
    """Low-rank adapters of every expert, trained beside its frozen weight: a slot's adapter is its expert's."""
    T, k, E, K, H, r = 60, 2, 4, 128, 96, 8
    up, _ = _layer(E, K, H, True)
    g = torch.Generator().manual_seed(4)
    x, ids = torch.randn((T, K), generator=g).bfloat16().cuda(), ids_of(T, k, E)
    a, b = (torch.randn((E, r, K), generator=g) / K ** 0.5).bfloat16().cuda(), (torch.randn((E, H, r), generator=g) / r ** 0.5).bfloat16().cuda()
    scales = torch.ones(E, device="cuda")
    place, token, begin = X.nvfp4_experts_sort(ids, E)
    slots = torch.arange(T * k, device="cuda")
    which = (torch.searchsorted(begin.long(), slots, right=True) - 1).to(torch.int32)          # E: behind the last expert's
    xs = X.nvfp4_experts_spread(x, place)
    h = X.experts_fprop(xs, begin, up)
    out = F.nvfp4_adapters_forward(xs, h, a, b, which, scales)
    for e in range(E):
        s = slice(int(begin[e]), int(begin[e + 1]))
        inner = xs[s].double() @ a[e].double().T
        ref = h[s].double() + inner @ b[e].double().T
        size = (xs[s].double().abs() @ a[e].double().abs().T) @ b[e].double().abs().T
        off = 2 * (K + r + 64) * U * size + 2.0 ** -16 * size
        close(out[s], ref, off + 2.0 ** -8 * (ref.abs() + off) + 1e-30, e)
    assert torch.equal(out[int(begin[E]):], h[int(begin[E]):])


def test_recovering_with_activations_as_they_are():
    """The example runs with unquantized activations too, and its gradients are finite and change the adapters."""
    from paper_2512_02010_amd import recover
    losses, adapted, plain = recover.run(steps=3, weight_only=True)
    assert all(v == v and 0 <= v < 1e3 for v in losses) and adapted == adapted and plain == plain


def test_without_tokens_and_without_rows():
    """A batch of no tokens goes through the layer and back; rows of out whose x has no rows at all are 0."""
    E, K, H, k = 3, 64, 96, 2
    up, down = _layer(E, K, H, True)
    x, ids, w = torch.empty((0, K), dtype=torch.bfloat16, device="cuda"), torch.empty((0, k), dtype=torch.int64, device="cuda"), torch.empty((0, k), device="cuda")
    y, kept = X.feed_forward(x, ids, w, up, down)
    dx, dw = X.feed_forward_backward(y, kept, w, up, down)
    assert y.shape == dx.shape == (0, K) and dw.shape == (0, k) and kept[1].tolist() == [0] * (E + 1)
    token, begin = torch.zeros(500, dtype=torch.int32, device="cuda"), torch.tensor([0, 5, 300, 400], dtype=torch.int32, device="cuda")
    ys = X.experts_fprop(x, begin, up, token)
    assert ys.shape == (500, H) and not bool(ys.any())

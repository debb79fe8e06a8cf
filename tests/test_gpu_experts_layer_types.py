"""GPU: a layer of experts with fp32 rows, which stay fp32 from product to product, and with infinities in masked places; against its definition in 64 bits,
step by step from what the step before left.  Bounds: sums of n products 2 n u (u = 2^-24; of fp32 rows three terms each and up to 64 partial sums), then
half a step of fp32, u."""
import pytest
import torch

from paper_2512_02010_amd import experts as X

from .test_gpu_experts import ids_of
from .test_gpu_experts_layer import _layer, _weights
from .test_gpu_weight_product import U, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T, k, E, K, H, block2d", [(1, 2, 4, 64, 96, True), (40, 3, 8, 128, 160, False), (900, 4, 6, 256, 512, True)])
def test_rows_of_fp32_stay_fp32(T, k, E, K, H, block2d):
    up, down = _layer(E, K, H, block2d)
    g = torch.Generator().manual_seed(2)
    x, dy = (torch.randn((T, K), generator=g).cuda() for _ in range(2))
    ids, weights = ids_of(T, k, E), torch.rand((T, k), generator=g).cuda()
    y, kept = X.feed_forward(x, ids, weights, up, down, base=x)
    place, begin, h, ys = kept
    assert {t.dtype for t in (y, h, ys)} == {torch.float32}
    b, there = begin.tolist(), place >= 0
    token = torch.zeros(T * k, dtype=torch.int64, device="cuda")
    token[place[there].long()] = torch.arange(T, device="cuda")[:, None].expand(T, k)[there]

    def off_of(n, size, ref):
        off = 2 * (3 * n + 64) * U * size + 2 * U * ref.abs()
        return off + U * (ref.abs() + off) + 1e-30

    wu, wd = _weights(up), _weights(down)
    for e in range(E):
        s = slice(b[e], b[e + 1])
        for got, source, w, n in ((h, x[token[s]], wu, K), (ys, torch.relu(h[s]), wd, H)):
            ref = source.double() @ w[e].T
            close(got[s], ref, off_of(n, source.double().abs() @ w[e].abs().T, ref), e)
    ref, size = x.double(), x.double().abs()
    for j in range(k):
        part = (weights[:, j] * there[:, j])[:, None].double() * ys[place[:, j].clamp(min=0).long()].double()
        ref, size = ref + part, size + part.abs()
    close(y, ref, (k + 3) * U * size + 1e-30, "y")

    dx, dw = X.feed_forward_backward(dy, kept, weights, up, down)
    assert dx.dtype == dw.dtype == torch.float32
    for j in range(k):
        products = dy.double() * ys[place[:, j].clamp(min=0).long()].double() * there[:, j, None]
        assert bool(((dw[:, j].double() - products.sum(1)).abs() <= (K + 1) * U * products.abs().sum(1)).all())
    ud, uu = _weights(down, True), _weights(up, True)
    ref, off = torch.zeros((T, K), dtype=torch.float64, device="cuda"), torch.zeros((T, K), dtype=torch.float64, device="cuda")
    for j in range(k):
        mine = there[:, j].nonzero()[:, 0]
        slot, e_of = place[mine, j].long(), ids[mine, j].long()
        for e in e_of.unique().tolist():
            t, s = mine[e_of == e], slot[e_of == e]
            dys = weights[t, j, None].double() * dy[t].double()
            d_off = U * dys.abs()
            mask = h[s] > 0
            dh = (dys @ ud[e]) * mask
            h_off = (d_off @ ud[e].abs() + off_of(K, (dys.abs() + d_off) @ ud[e].abs(), dh)) * mask
            dxs = dh @ uu[e]
            ref[t] += dxs
            off[t] += h_off @ uu[e].abs() + off_of(H, (dh.abs() + h_off) @ uu[e].abs(), dxs) + (k + 2) * U * dxs.abs()
    close(dx, ref, off + U * (ref.abs() + off) + 1e-30, "dx")


@pytest.mark.parametrize("dtype, other", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_a_base_of_another_type(dtype, other):
    """The result has base's type, dx that of dy, the rows in between x's: the same numbers, rounded once more or not."""
    T, k, E, K, H = 70, 2, 5, 96, 64
    up, down = _layer(E, K, H, True)
    g = torch.Generator().manual_seed(3)
    x, base, dy = (torch.randn((T, K), generator=g).bfloat16().cuda() for _ in range(3))
    x, ids, weights = x.to(dtype), ids_of(T, k, E), torch.rand((T, k), generator=g).cuda()
    made = {}
    for t in (dtype, other):
        y, kept = X.feed_forward(x, ids, weights, up, down, base=base.to(t))
        dx, dw = X.feed_forward_backward(dy.to(t), kept, weights, up, down)
        assert y.dtype == dx.dtype == t and kept[2].dtype == kept[3].dtype == dtype
        made[t] = y, dx, kept[2], kept[3], dw
    for a, b in zip(made[torch.float32][:2], made[torch.bfloat16][:2]):
        assert torch.equal(a.bfloat16(), b)
    assert all(torch.equal(a, b) for a, b in zip(made[dtype][2:], made[other][2:]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [3, 200])
def test_infinities_behind_the_activation_do_not_come_through(T, dtype):
    """Where the activation is cut off its gradient is 0, also of a gradient that has overflowed: a token whose hidden columns are all negative
    gets none, whatever comes back to it."""
    E, K, H, k = 3, 64, 96, 2
    g = torch.Generator().manual_seed(4)
    up = X.quantize_experts((0.5 + torch.rand((E, H, K), generator=g)).cuda())
    down = X.quantize_experts(torch.randn((E, K, H), generator=g).cuda())
    x, dy = ((0.5 + torch.rand((T, K), generator=g)).to(dtype).cuda() for _ in range(2))
    x[1] *= -1                                     # (positive weights: all of its hidden columns are negative, all others' positive)
    ids, w = torch.randint(0, E, (T, k), generator=g).cuda(), 0.5 + torch.rand((T, k), generator=g).cuda()
    y, kept = X.feed_forward(x, ids, w, up, down)
    assert not bool(y[1].any())
    want, _ = X.feed_forward_backward(dy, kept, w, up, down)
    assert not bool(want[1].any()) and bool(want[0].any())
    for bad in (float("inf"), float("-inf"), float("nan")):
        dy[1] = bad
        dx, _ = X.feed_forward_backward(dy, kept, w, up, down)
        assert torch.equal(dx, want), bad

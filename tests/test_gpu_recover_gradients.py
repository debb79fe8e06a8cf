"""GPU: the recovering example with unquantized activations (``weight_only``): every adapter has a gradient that moves it, and a layer's results and
gradients are their formulas'.

Bounds (u = 2^-24, half a step of BF16 2^-8): the projection is a sum of n exact products, 2 (n + 64) u of the magnitudes, rounded to BF16; on top of it comes
the adapter's part, h (or dh) in two BF16 terms, of which 2^-16 is left, in sums of n products each, then BF16 again."""
import pytest
import torch

from paper_2512_02010_amd import recover

from .test_gpu_weight_product import U, close, values

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def test_every_adapter_learns(monkeypatch):
    made = []

    class Watched(recover.AdaptedLinear):
        def __init__(self, *args):
            super().__init__(*args)
            assert self.weight_only
            self.first, self.seen = [t.clone() for t in self.master], []
            made.append(self)

        def backward(self, *args, **kw):
            dx = super().backward(*args, **kw)
            self.seen.append([g.clone() for g in self.grads])
            return dx

    monkeypatch.setattr(recover, "AdaptedLinear", Watched)
    recover.run(steps=3, weight_only=True)
    assert len(made) == 3
    for layer in made:
        assert len(layer.seen) == 3 and all(bool(g.isfinite().all()) for step in layer.seen for g in step)
        # B is 0 at first, and so is A's first gradient; from then on neither of any adapter is
        assert not bool(layer.seen[0][0].any()) and all(bool(g[i].any()) for step in layer.seen[1:] for g in step for i in range(2))
        assert all(bool((now[i] != before[i]).any()) for now, before in zip(layer.master, layer.first) for i in range(2))


@pytest.mark.parametrize("T", [7, 300])
def test_a_layer_and_its_gradients(T):
    N, K, r = 160, 96, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    layer = recover.AdaptedLinear(normal(N, K), 2, r, g, True)
    layer.master[1] = normal(2, N, r)
    layer.cast()
    x, dy = normal(T, K).bfloat16(), normal(T, N).bfloat16()
    which = torch.randint(-1, 2, (T,), generator=g, device="cuda", dtype=torch.int32)
    y, dx = layer.forward(x, which, True), None
    dx = layer.backward(dy, 0)
    q = layer.quantized
    w = q["alpha"].double() * values(q["codes_row"], q["scales_row"], q["block2d"])
    X, D = x.double(), dy.double()
    for i in range(-1, 2):
        t = (which == i).nonzero()[:, 0]
        a, b = (layer.a[i].double(), layer.b[i].double()) if i >= 0 else (X.new_zeros((r, K)), X.new_zeros((N, r)))
        for got, source, weight, one, two, n in ((y, X[t], w.T, a.T, b.T, K), (dx, D[t], w, b, a, N)):
            base, inner, size = source @ weight, source @ one @ two, source.abs() @ one.abs() @ two.abs()
            off = 2 * (n + 64) * U * (source.abs() @ weight.abs()) + 2 * U * base.abs()
            off = off + HALF * (base.abs() + off) + (2 * (n + r + 64) * U + 2.0 ** -16) * size
            ref = base + inner
            close(got[t], ref, off + HALF * (ref.abs() + off) + 1e-30, i)
        if i >= 0:
            da, db = (v[i] for v in layer.grads)
            for got, ref, size, n in ((da, (D[t] @ b).T @ X[t], (D[t].abs() @ b.abs()).T @ X[t].abs(), N),
                                      (db, D[t].T @ (X[t] @ a.T), D[t].abs().T @ (X[t].abs() @ a.abs().T), K)):
                # (dh or h in fp32, then in two BF16 terms, summed over the tokens)
                close(got, ref, (2 * (n + len(t) + 64) * U + 2.0 ** -16) * size + 1e-30, i)

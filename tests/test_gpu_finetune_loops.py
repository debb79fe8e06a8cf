"""GPU: adapters and distillation at the sizes where their kernels go through their loops (several tiles, adapters or rows a
workgroup), against the definitions in 64 bits, with the tolerances of test_gpu_adapters.py and test_gpu_distill.py."""
import pytest
import torch

from paper_2512_02010_amd import finetune as F

from . import _finetune_sizes as sizes
from .test_gpu_adapters import _check_backward, _check_forward, _which
from .test_gpu_distill import _check, _inputs

pytestmark = pytest.mark.gpu


def _adapters(T, K, N, r, adapters, order, dtype=torch.bfloat16, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    return dict(x=(normal(T, K) * torch.exp(normal(T, 1))).bfloat16(), a=(normal(adapters, r, K) / K ** 0.5).bfloat16(),
                b=(normal(adapters, N, r) / r ** 0.5).bfloat16(), which=_which(T, adapters, order, seed).cuda(),
                scales=0.25 + 2 * torch.rand(adapters, generator=g, device="cuda"), base=normal(T, N).to(dtype),
                dy=(1e-3 * normal(T, N) * torch.exp(normal(T, 1))).bfloat16(), dx_base=(1e-3 * normal(T, K)).bfloat16())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,K,N,r,adapters,order", sizes.ADAPTERS + sizes.ADAPTERS_FEW)
def test_adapters_forward(T, K, N, r, adapters, order, dtype):
    s = _adapters(T, K, N, r, adapters, order, dtype)
    out, h = _check_forward(s, dtype)
    base = s["base"].clone()
    in_place = F.nvfp4_adapters_forward(s["x"], base, s["a"], s["b"], s["which"], s["scales"], out=base)
    assert in_place.data_ptr() == base.data_ptr() and torch.equal(in_place, out)


@pytest.mark.parametrize("T,K,N,r,adapters,order", sizes.ADAPTERS + sizes.ADAPTERS_FEW)
def test_adapters_backward(T, K, N, r, adapters, order):
    s = _adapters(T, K, N, r, adapters, order)
    _, h = F.nvfp4_adapters_forward(s["x"], None, s["a"], s["b"], s["which"], s["scales"], want_h=True)
    dx, da, db = _check_backward(s, h=h)
    base = s["dx_base"].clone()
    again = F.nvfp4_adapters_backward(s["dy"], s["x"], h, s["a"], s["b"], s["which"], s["scales"], base, out=base)
    for u, v in zip(again, (dx, da, db)):
        assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,V,k", sizes.DISTILL)
def test_distillation(T, V, k, dtype):
    s = _inputs(T, V // 2 if dtype == torch.float32 else V, k, dtype)
    s["index"][::3, k // 2:] = s["index"][::3, :1]          # one word again and again, also in lists that have nothing else
    loss, lse, d, step_loss, step_d = _check(s, tau=1.5)
    args = (s["logits"], s["teacher"], s["index"])
    logits = s["logits"].clone()
    out = F.nvfp4_distill_backward(logits, *args[1:], lse, s["weight"], 1.5, out=logits)
    assert out.data_ptr() == logits.data_ptr() and torch.equal(out, d)
    logits.copy_(s["logits"])
    again, out = F.nvfp4_distill_step(logits, *args[1:], s["weight"], 1.5, out=logits)
    assert out.data_ptr() == logits.data_ptr() and torch.equal(out, step_d) and torch.equal(again, step_loss)

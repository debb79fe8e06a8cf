"""GPU: offsets past 32 bits, in elements and in bytes, of every operand that can be so large, against the same calls on the parts that lie there."""
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import experts as X

from .test_gpu_weight_product import rows, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N, K", [(48, 64), (520, 96)])
def test_rows_far_apart(N, K):
    """x and the result with strides that put their last rows beyond 2^32 elements: in tiles of rows, and gathered a few at a time."""
    T, ld = 70000, 65536
    codes, scales, alpha = weights(1, N, K, False)
    room = torch.empty((T, ld), dtype=torch.bfloat16, device="cuda")
    assert room.numel() > 1 << 32
    x, out = room[:, 64:64 + K], room[:, 1024:1024 + N]
    x.copy_(rows(T, K, torch.bfloat16))
    want = X.nvfp4_weight_product(x.contiguous(), codes[0], scales[0], alpha)
    X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out=out)
    assert torch.equal(out, want)
    token = torch.tensor([T - 1, 0, T - 2], dtype=torch.int32, device="cuda")
    begin = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    few = X.nvfp4_experts_product(x, begin, codes, scales, alpha, token=token)
    assert torch.equal(few, X.nvfp4_weight_product(x[token.long()].contiguous(), codes[0], scales[0], alpha))


def test_experts_whose_codes_pass_32_bits():
    E, N, K = 1024, 4096, 2304
    codes = torch.randint(0, 256, (E, N, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.randint(0, 127, (E, N, K // 16), dtype=torch.uint8, device="cuda")
    assert codes.numel() > 1 << 32
    alpha = 0.5 + torch.rand(E, device="cuda")
    for last in (2, 300):                              # rows of the last expert: few, and in tiles
        x = rows(last + 1, K, torch.bfloat16)
        begin = torch.ones(E + 1, dtype=torch.int32, device="cuda")
        begin[0], begin[E] = 0, last + 1
        ys = X.nvfp4_experts_product(x, begin, codes, scales, alpha, out_dtype=B.OUT_F32)
        for e, s in ((0, slice(0, 1)), (E - 1, slice(1, last + 1))):
            one = X.nvfp4_weight_product(x[s], codes[e], scales[e], alpha[e:e + 1], out_dtype=B.OUT_F32)
            # (another order of the same exact products: 2 K u of their magnitudes each)
            size = X.nvfp4_weight_product(x[s].abs(), codes[e] & 0x77, scales[e], alpha[e:e + 1], out_dtype=B.OUT_F32)
            assert bool(((ys[s] - one).abs() <= 2 * 2 * (K + 64) * 2.0 ** -24 * 1.001 * size).all())


def test_places_whose_rows_pass_32_bits():
    T, k, W = 9000, 64, 8192
    assert T * k * W > 1 << 32
    ids = torch.randint(-1, 1000, (T, k), dtype=torch.int64, device="cuda")
    place, token, begin = X.nvfp4_experts_sort(ids, 1000)
    x = torch.randn((T, W), device="cuda").bfloat16()
    xs = X.nvfp4_experts_spread(x, place)
    for first in range(0, T * k, 1 << 16):             # (a part at a time)
        t = token[first:first + (1 << 16)]
        assert torch.equal(xs[first:first + (1 << 16)], torch.where((t >= 0)[:, None], x[t.clamp(min=0).long()], 0))
    part = slice(T - 64, T)
    small = torch.arange(64 * k, dtype=torch.int32, device="cuda").reshape(64, k)          # the same rows, near by
    slot = torch.where(place[part] >= 0, place[part], ~place[part]).flatten().long()
    near, there = torch.where(place[part] >= 0, small, ~small), xs[slot]
    w = torch.rand((T, k), device="cuda")
    assert torch.equal(X.nvfp4_experts_combine(xs, place, w)[part], X.nvfp4_experts_combine(there, near, w[part]))
    dys, dw = X.nvfp4_experts_combine_backward(x, xs, place, w, out=xs)
    dys2, dw2 = X.nvfp4_experts_combine_backward(x[part], there, near, w[part])
    assert torch.equal(dys[slot], dys2) and torch.equal(dw[part], dw2)

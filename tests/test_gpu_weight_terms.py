"""fp32 activations enter the products with all 24 bits: every one of their three BF16 terms counts, in every kernel.

Each row of x has one number, whose last bits are not 0; weights without alpha and alpha are powers of two.  So the sum that a result is has one term and
the result is exact: in fp32 it has all 24 bits, in BF16 the last of them says to which side of a tie it is.  Nothing rounds before that, so
results have to be equal.  (Sizes as in the tests of the products, which reach every kernel.)"""
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import experts as X

from .test_gpu_weight_product import EXPERTS, SIZES, _routed, values

POWERS = (1, 2, 4, 6, 9, 10, 12, 14)             # codes of 0.5, 1, 2, 4 and the same below 0
BF16, F32 = torch.bfloat16, torch.float32


def numbers(n, out_dtype, g):
    """n fp32 numbers whose last eight bits decide the result: all 24 bits at random, but the ninth and the last 1 (so that the second term has the middle eight
    and the third is not 0), or, for a BF16 result, a tie of an even number and the next but for the last bit."""
    bits = torch.randint(0, 1 << 23, (n,), generator=g, dtype=torch.int32)
    bits = bits | 0x8001 if out_dtype == F32 else bits & 0x7e0000 | 0x8001
    exponent = torch.randint(107, 147, (n,), generator=g, dtype=torch.int32)
    sign = torch.randint(0, 2, (n,), generator=g, dtype=torch.int32) << 31
    return (bits | exponent << 23 | sign).view(F32)


def one_each(T, K, out_dtype, seed):
    """x [T][K] of one number in every row, and where it stands: at the ends of K, then anywhere."""
    g = torch.Generator().manual_seed(seed)
    at = torch.randint(0, K, (T,), generator=g)
    ends = [K - 1, 0, K - 32, K - 17, K // 2]
    at[seed % T] = ends[seed % len(ends)]
    x = torch.zeros((T, K))
    x[torch.arange(T), at] = numbers(T, out_dtype, g)
    return x, at


def powers(E, N, K, tiles):
    g = torch.Generator().manual_seed(7)
    kinds = torch.tensor(POWERS, dtype=torch.uint8)
    draw = lambda: kinds[torch.randint(0, 8, (E, N, K // 2), generator=g)]          # noqa: E731
    codes = draw() | draw() << 4
    scales = 8 * torch.randint(1, 15, (E, N // 16 if tiles else N, K // 16), generator=g).to(torch.uint8)
    alpha = 2.0 ** -torch.arange(E).remainder(5).float()
    return codes.cuda(), scales.cuda(), alpha.cuda()


@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_two_terms_are_not_enough(out_dtype):
    """CPU: what the first two terms of these numbers come to is another result for every one of them."""
    x = numbers(10000, out_dtype, torch.Generator().manual_seed(1))
    first = (x.view(torch.int32) & -65536).view(F32)
    second = ((x - first).view(torch.int32) & -65536).view(F32)
    third = x - first - second
    assert torch.equal(third, ((x - first - second).view(torch.int32) & -65536).view(F32)) and torch.equal(third + second + first, x)
    for w in (0.5, -4.0, 2.0 ** -11):
        assert bool(((x * w).to(out_dtype) != ((first + second) * w).to(out_dtype)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("T, K, N, tiles", SIZES)
def test_one_weight(T, K, N, tiles, out_dtype):
    codes, scales, alpha = powers(1, N, K, tiles)
    w = values(codes[0], scales[0], tiles)
    for seed in range(8 if T < 20 else 2):
        x, at = one_each(T, K, out_dtype, seed)
        y = X.nvfp4_weight_product(x.cuda(), codes[0], scales[0], alpha, out_dtype=int(out_dtype == F32), flags=B.GEMM_B_TILE_SCALES if tiles else 0)
        want = x.sum(1).double().cuda()[:, None] * w[:, at.cuda()].T * alpha.double()
        assert torch.equal(y, want.to(F32).to(out_dtype)), seed


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("T, k, E, K, N, tiles", EXPERTS)
def test_experts(T, k, E, K, N, tiles, out_dtype):
    codes, scales, alpha = powers(E, N, K, tiles)
    _, token, begin = X.nvfp4_experts_sort(_routed(T, k, E), E)
    x, at = one_each(T, K, out_dtype, T)
    xc, at, b = x.cuda(), at.cuda(), begin.tolist()
    ys = X.nvfp4_experts_product(xc, begin, codes, scales, alpha, token=token, out_dtype=int(out_dtype == F32), flags=B.GEMM_B_TILE_SCALES if tiles else 0)
    number = xc.sum(1).double()
    for e in range(E):
        t = token[b[e]:b[e + 1]].long()
        if len(t):
            want = number[t][:, None] * values(codes[e], scales[e], tiles)[:, at[t]].T * alpha[e].double()
            assert torch.equal(ys[b[e]:b[e + 1]], want.to(F32).to(out_dtype)), e
    assert not bool(ys[b[E]:].any())

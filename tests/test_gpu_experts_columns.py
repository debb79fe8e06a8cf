"""GPU: as many experts and columns as the header allows, so that a workgroup for every tile that there might be would be more than a launch has: 75 GB of
weights, three rows of 2^22 columns for each of a thousand experts."""
import pytest
import torch

from paper_2512_02010_amd import experts as X

from .test_gpu_weight_product import bound, close, rows, values

pytestmark = pytest.mark.gpu


def test_a_thousand_experts_of_four_million_columns():
    E, N, K, S = 1000, 1 << 22, 32, 3000
    codes = torch.empty(E * N * K // 2 // 8, dtype=torch.int64, device="cuda").random_().view(torch.uint8).view(E, N, K // 2)
    scales = torch.randint(0, 127, (E, N, K // 16), dtype=torch.uint8, device="cuda")
    alpha, x = (0.5 + torch.rand(E, device="cuda")) / K, rows(S, K, torch.bfloat16)
    b = [min(3 * e, S - 6) for e in range(E)] + [S - 2]                    # (one expert without rows, the last with four, two rows behind them)
    begin = torch.tensor(b, dtype=torch.int32, device="cuda")
    out = torch.full((S, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    X.nvfp4_experts_product(x, begin, codes, scales, alpha, out=out)
    for e in (0, 1, 500, 997, 998, 999):
        for n in (slice(0, 300), slice(N // 2 - 100, N // 2 + 100), slice(N - 260, N)):
            w, mine = values(codes[e, n], scales[e, n], False), x[b[e]:b[e + 1]]
            ref = alpha[e].double() * (mine.double() @ w.T)
            close(out[b[e]:b[e + 1], n], ref, bound(mine, w, alpha[e], ref, torch.bfloat16, torch.bfloat16), (e, n))
    assert not bool(out[b[E]:].any())
    for first in range(0, S, 250):                                          # every element was written
        assert not bool(out[first:first + 250].isnan().any())
    del codes, scales, out
    torch.cuda.empty_cache()

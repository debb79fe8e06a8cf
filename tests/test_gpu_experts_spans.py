"""GPU: rows that no expert has, in front of the first one's and behind the last one's, are 0: of a span of the experts, whose begins do not start at 0."""
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import experts as X

from .test_gpu_weight_product import bound, close, rows, values, weights

pytestmark = pytest.mark.gpu

SIZES = [  # rows, experts, K, N: few rows for each expert, tiles of each kind, one expert alone
    (1, 1, 32, 1), (9, 1, 96, 40), (5, 4, 64, 40), (40, 64, 1024, 72), (90, 4, 64, 40), (200, 16, 288, 100), (700, 4, 64, 513), (900, 1, 256, 300),
    (1500, 3, 512, 1040), (6000, 3, 128, 2048),
]


def _begins(S, E):
    """Of spans that leave out rows in front, behind, on both sides, or all rows."""
    third = S // 3
    inner = [third + i * (S - 2 * third) // E for i in range(E + 1)]
    return [inner, [third + (i > E // 2) * (S - third) for i in range(E + 1)], [S] * (E + 1), [third] * (E + 1), [0] * (E + 1),
            [min(1, S)] + [S - 1] * E]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("S, E, K, N", SIZES)
def test_rows_without_an_expert_are_zero(S, E, K, N, dtype):
    (codes, scales, alpha), x = weights(E, N, K, False), rows(S, K, dtype)
    for b in _begins(S, E):
        begin = torch.tensor(b, dtype=torch.int32, device="cuda")
        room = torch.full((S, N + 8), float("nan"), dtype=dtype, device="cuda")
        out = X.nvfp4_experts_product(x, begin, codes, scales, alpha, out=room[:, :N])
        for e in range(E):
            mine, w = x[b[e]:b[e + 1]], values(codes[e], scales[e], False)
            ref = alpha[e].double() * (mine.double() @ w.T)
            close(out[b[e]:b[e + 1]], ref, bound(mine, w, alpha[e], ref, dtype, dtype), (b, e))
        assert bool((out[:b[0]] == 0).all()) and bool((out[b[E]:] == 0).all()), b
        assert bool(room[:, N:].isnan().all())


def test_a_span_of_the_experts():
    """The products of the experts 3 .. 6 of eight, by the part of `begin` that is theirs: all others' rows are 0."""
    for T in (6, 150, 3000):
        E, k, K, N = 8, 2, 256, 144
        g = torch.Generator().manual_seed(T)
        ids = torch.randint(-1, E, (T, k), generator=g).cuda()
        place, token, begin = X.nvfp4_experts_sort(ids, E)
        (codes, scales, alpha), x = weights(E, N, K, True), rows(T, K, torch.bfloat16)
        all_ = X.nvfp4_experts_product(x, begin, codes, scales, alpha, token=token, flags=B.GEMM_B_TILE_SCALES)
        some = X.nvfp4_experts_product(x, begin[3:8].clone(), codes[3:7], scales[3:7], alpha[3:7].clone(), token=token, flags=B.GEMM_B_TILE_SCALES)
        first, last = int(begin[3]), int(begin[7])
        for e in range(3, 7):
            s = slice(int(begin[e]), int(begin[e + 1]))
            w, mine = values(codes[e], scales[e], True), x[token[s].long()]
            ref = alpha[e].double() * (mine.double() @ w.T)
            off = bound(mine, w, alpha[e], ref, torch.bfloat16, torch.bfloat16)
            close(some[s], ref, off, (T, e))
            close(all_[s], ref, off, (T, e))
        assert not bool(some[:first].any()) and not bool(some[last:].any())


def test_begins_that_fall_over_a_billion_rows():
    """Every other expert claims all rows: their tiles, added up, pass 32 bits.  No result is promised, but nothing outside the result is
    written (its margins are checked after the test)."""
    S, E, K, N = 1 << 30, 1024, 32, 1
    (codes, scales, alpha), x = weights(E, N, K, False), rows(8, K, torch.bfloat16)
    token = torch.full((S,), 3, dtype=torch.int32, device="cuda")
    for b in ([0, S] * 512 + [0], [S, 0] * 512 + [S], [S // 2, S, 0, S] * 256 + [S // 4]):
        begin = torch.tensor(b, dtype=torch.int32, device="cuda")
        assert X.nvfp4_experts_product(x, begin, codes, scales, alpha, token=token).shape == (S, N)
        torch.cuda.synchronize()

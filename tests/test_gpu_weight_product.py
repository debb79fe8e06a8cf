"""GPU: products of unquantized activations with NVFP4 weights, one or one for each expert, against their definition in 64 bits.

Tolerances, per element, from the arithmetic alone (u = 2^-24, fp32's half unit): a weight's value without alpha is exact, an fp32 activation is three
terms exactly, and so are the products; a sum of n of them in any order is within 2 n u of the sum of magnitudes (the factor 2 for the matrix unit's
truncation), n = K or 3 K and up to 64 partial sums; then alpha, u, and the rounding to the output's type, half a step.
"""
import numpy as np
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import experts as X
from paper_2512_02010_amd import linear as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -140                    # BF16 terms of an fp32 number end at 2^-133, times weights of up to 2^11
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def weights(E, N, K, tiles, seed=1):
    """Codes of every kind, scales of every byte that there is (subnormals and 0 too); both as the library lays them out."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (E, N, K // 2), generator=g, dtype=torch.uint8)
    scales = torch.randint(0, 127, (E, N // 16 if tiles else N, K // 16), generator=g, dtype=torch.uint8)
    alpha = (0.25 + torch.rand(E, generator=g)) / K
    return codes.cuda(), scales.cuda(), alpha.cuda()


def values(codes, scales, tiles):
    """[N][K] in 64 bits, without alpha"""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device=codes.device)
    c = torch.stack(((codes & 15).long(), (codes >> 4).long()), 2).flatten(1)
    s = scales.view(torch.float8_e4m3fn).double().repeat_interleave(16, 1)
    return grid[c] * (s.repeat_interleave(16, 0) if tiles else s)


def rows(T, K, dtype, seed=2):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, K), generator=g) * torch.exp(torch.randn((T, 1), generator=g))).to(dtype).cuda()


def bound(x, w, alpha, ref, dtype, out_dtype):
    n = (3 if dtype == torch.float32 else 1) * x.shape[1] + 64
    off = float(alpha) * (2 * n * U * (x.double().abs() @ w.abs().T) + TINY) + 2 * U * ref.abs()
    half = 2.0 ** -8 if out_dtype == torch.bfloat16 else U
    return off + half * (ref.abs() + off) + 1e-37


def close(got, ref, off, what=""):
    bad = (got.double() - ref).abs() > off
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got.double() - ref).abs() / off).max()))


SIZES = [  # T, K, N, tiles
    (1, 32, 1, False), (1, 32, 16, True), (1, 4096, 4096, False), (1, 160, 33, False), (2, 64, 48, True), (3, 2880, 1440, True), (5, 8192, 1000, False),
    (15, 1056, 17, False), (16, 128, 2048, True), (17, 1024, 512, False), (24, 2048, 2048, True), (33, 96, 100, False), (48, 4096, 528, True),
    (64, 512, 4096, False), (65, 544, 130, False), (100, 2048, 1024, True), (127, 256, 257, False), (128, 1024, 1024, False),
    (129, 1056, 336, True), (200, 4096, 304, True), (255, 128, 511, False), (256, 8192, 256, False), (300, 32, 2000, False), (513, 992, 1008, True),
    (1000, 2048, 2049, False), (1025, 1024, 3008, True), (2049, 608, 1023, False),
    (2, 256, 100, False), (4, 96, 64, True), (6, 512, 72, False), (7, 224, 60, False), (9, 256, 40, False), (12, 96, 300, False), (13, 768, 144, True),
    (48, 512, 8192, False), (60, 96, 1000, False), (300, 2048, 4096, True), (2049, 608, 4096, False), (4096, 256, 4096, True),
    (4000, 1056, 3000, False), (500, 4096, 9001, False), (3900, 2080, 4096, True),
]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T, K, N, tiles", SIZES)
def test_one_weight(T, K, N, tiles, dtype, out_dtype):
    (codes, scales, alpha), x = weights(1, N, K, tiles), rows(T, K, dtype)
    y = X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out_dtype=int(out_dtype == torch.float32),
                               flags=B.GEMM_B_TILE_SCALES if tiles else 0)
    assert y.shape == (T, N) and y.dtype == out_dtype
    w = values(codes[0], scales[0], tiles)
    ref = alpha.double() * (x.double() @ w.T)
    close(y, ref, bound(x, w, alpha, ref, dtype, out_dtype))
    assert torch.equal(y, X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out=torch.empty_like(y),
                                                 flags=B.GEMM_B_TILE_SCALES if tiles else 0))


@pytest.mark.parametrize("T", [1, 20, 150, 700])
def test_strides(T):
    """Rows of x and of the result a stride apart; what lies between the result's rows stays."""
    codes, scales, alpha = weights(1, 200, 256, False)
    x = rows(T, 512, torch.bfloat16)[:, 128:384]
    for pad in (0, 1, 24):                             # (an odd stride too)
        room = torch.full((T, 200 + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out=room[:, :200])
        assert torch.equal(room[:, :200], X.nvfp4_weight_product(x.contiguous(), codes[0], scales[0], alpha))
        assert bool((room[:, 200:] == 7).all())


def test_no_rows():
    codes, scales, alpha = weights(1, 64, 64, False)
    assert X.nvfp4_weight_product(rows(0, 64, torch.bfloat16), codes[0], scales[0], alpha).shape == (0, 64)


@pytest.mark.parametrize("T", [3, 40, 300])
def test_quantized_by_the_library(T):
    """Both packings of a weight that the library quantized, against its own dequantization: x W^T and dy W."""
    N, K = 544, 288
    for block2d in (False, True):
        g = torch.Generator().manual_seed(5)
        q = L.quantize_weight(torch.randn((N, K), generator=g).cuda(), block2d=block2d)
        flags = B.GEMM_B_TILE_SCALES if block2d else 0
        for x, codes, scales in ((rows(T, K, torch.bfloat16), q["codes_row"], q["scales_row"]),
                                 (rows(T, N, torch.bfloat16), q["codes_col"], q["scales_col"])):
            w = values(codes, scales, block2d)
            ref = q["alpha"].double() * (x.double() @ w.T)
            close(X.nvfp4_weight_product(x, codes, scales, q["alpha"], flags=flags), ref,
                  bound(x, w, q["alpha"], ref, torch.bfloat16, torch.bfloat16))
        if block2d:                                     # the same values in both
            assert torch.equal(values(q["codes_row"], q["scales_row"], True), values(q["codes_col"], q["scales_col"], True).T)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [4, 90, 400])
def test_infinities_and_nan(T, dtype):
    """As fp32 arithmetic has them, and only in their own rows: inf times 0 is NaN, inf times what is not 0 is inf."""
    K, N = 160, 70
    (codes, scales, alpha), x = weights(1, N, K, False), rows(T, K, dtype)
    w = values(codes[0], scales[0], False)
    clean = X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out_dtype=B.OUT_F32)
    x[1, 7], x[2, 100] = float("inf"), float("nan")
    got = X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out_dtype=B.OUT_F32)
    rest = [i for i in range(T) if i not in (1, 2)]
    assert torch.equal(got[rest], clean[rest]) and bool(got[2].isnan().all())
    zero = w[:, 7] == 0
    assert bool(got[1][zero].isnan().all()) and torch.equal(got[1][~zero], torch.sign(w[:, 7][~zero]).float() * float("inf"))
    # the type's largest numbers, and fp32's least
    big = torch.full((T, K), torch.finfo(dtype).max, dtype=dtype, device="cuda")
    small = torch.full((1, 32), 0x70, dtype=torch.uint8, device="cuda")
    one = torch.full((1, 16), 0x11, dtype=torch.uint8, device="cuda")           # 0.5 each
    y = X.nvfp4_weight_product(big[:, :32] * 2.0 ** -20, one, small[:, :2].contiguous(), torch.ones(1, device="cuda"), out_dtype=B.OUT_F32)
    ref = 32 * 0.5 * 128 * 2.0 ** -20 * float(torch.finfo(dtype).max)
    assert bool(((y.double() - ref).abs() <= 2 * 160 * U * ref).all())


def _routed(T, k, E, seed=3, none=0.1):
    r = np.random.default_rng(seed)
    ids = np.stack([r.permutation(E)[:k] if k <= E else r.integers(0, E, k) for _ in range(T)]).astype(np.int32)
    ids[r.random((T, k)) < none] = -1
    return torch.from_numpy(ids).cuda()


EXPERTS = [  # T, k, E, K, N, tiles
    (1, 1, 1, 32, 16, True), (1, 2, 4, 64, 100, False), (7, 3, 5, 160, 33, False), (32, 4, 64, 512, 256, True), (50, 2, 3, 1056, 144, True),
    (64, 8, 16, 256, 520, False), (200, 1, 200, 96, 40, False), (333, 2, 7, 288, 272, True), (600, 4, 8, 512, 500, False),
    (1500, 2, 2, 128, 384, True), (2000, 1, 1, 320, 64, False), (900, 6, 30, 224, 1040, True), (4000, 2, 3, 1024, 264, False),
    (20, 2, 4, 96, 250, False), (4, 2, 4, 256, 256, True), (3, 3, 8, 160, 72, False), (30, 2, 16, 512, 64, True), (100, 2, 1024, 64, 48, True),
    (4096, 4, 32, 2080, 2300, False), (6000, 2, 8, 128, 2048, True),
]


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("dtype, out_dtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32),
                                              (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T, k, E, K, N, tiles", EXPERTS)
def test_experts(T, k, E, K, N, tiles, dtype, out_dtype, gather):
    codes, scales, alpha = weights(E, N, K, tiles)
    _, token, begin = X.nvfp4_experts_sort(_routed(T, k, E), E)
    x = rows(T if gather else T * k, K, dtype)
    ys = X.nvfp4_experts_product(x, begin, codes, scales, alpha, token=token if gather else None,
                                 out_dtype=int(out_dtype == torch.float32), flags=B.GEMM_B_TILE_SCALES if tiles else 0)
    assert ys.shape == (T * k, N) and ys.dtype == out_dtype
    b = begin.tolist()
    for e in range(E):
        mine = x[token[b[e]:b[e + 1]].long()] if gather else x[b[e]:b[e + 1]]
        w = values(codes[e], scales[e], tiles)
        ref = alpha[e].double() * (mine.double() @ w.T)
        close(ys[b[e]:b[e + 1]], ref, bound(mine, w, alpha[e], ref, dtype, out_dtype), e)
    assert not bool(ys[b[E]:].any())


def _spans(x, b, codes, scales, alpha, token=None):
    return X.nvfp4_experts_product(x, torch.tensor(b, dtype=torch.int32, device="cuda"), codes, scales, alpha, token=token)


@pytest.mark.parametrize("S", [5, 60, 700])
def test_begins_and_tokens_that_are_wrong(S):
    """Whatever begin and token hold, only rows of x are read and rows of out written; a row without one of x's rows is 0."""
    E, K, N = 4, 64, 40
    (codes, scales, alpha), x = weights(E, N, K, False), rows(S, K, torch.bfloat16)
    right = _spans(x, [0, 2, 2, S - 1, S], codes, scales, alpha)
    huge = _spans(x, [-2 ** 31, 2, 2, S - 1, 2 ** 31 - 1], codes, scales, alpha)
    assert torch.equal(huge, right)
    _spans(x, [S, 2 ** 31 - 1, -5, S // 2, -2 ** 31], codes, scales, alpha)         # (falling: no result is promised)
    token = torch.arange(S, dtype=torch.int32, device="cuda")
    token[1], token[3], token[4] = -1, S, -2 ** 31
    got = _spans(x, [0, 2, 2, S - 1, S], codes, scales, alpha, token)
    keep = [i for i in range(S) if i not in (1, 3, 4)]
    assert torch.equal(got[keep], right[keep]) and not bool(got[[1, 3, 4]].any())
    assert not bool(_spans(x, [0] * 5, codes, scales, alpha).any())


def test_an_expert_alone_is_one_weight():
    """Up to the order of sums: the same products, of rows that all belong to one expert of several."""
    for T in (3, 70, 500):
        (codes, scales, alpha), x = weights(3, 136, 256, False), rows(T, 256, torch.bfloat16)
        w = values(codes[1], scales[1], False)
        ref = alpha[1].double() * (x.double() @ w.T)
        close(_spans(x, [0, 0, T, T], codes, scales, alpha), ref, bound(x, w, alpha[1], ref, torch.bfloat16, torch.bfloat16))
        one = X.nvfp4_weight_product(x, codes[1], scales[1], alpha[1:2])
        close(one, ref, bound(x, w, alpha[1], ref, torch.bfloat16, torch.bfloat16))


def test_on_another_stream():
    codes, scales, alpha = weights(1, 512, 512, False)
    x = rows(40, 512, torch.bfloat16)
    want = X.nvfp4_weight_product(x, codes[0], scales[0], alpha)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = X.nvfp4_weight_product(x, codes[0], scales[0], alpha, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def _in_two_graphs(call, inputs):
    """Captured twice, replayed in turn with new values in the same tensors, eager work of the program's own between them."""
    graphs = []
    for _ in range(2):
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        graphs.append((graph, got))
    for turn in range(3):
        for graph, got in graphs:
            for t in inputs:
                t.copy_(torch.roll(t, 1, 0))
            eager = call()
            graph.replay()
            assert torch.equal(got, eager), turn
            torch.cuda.synchronize()


@pytest.mark.parametrize("T", [1, 12, 40, 600])
def test_replayed_from_a_graph(T):
    codes, scales, alpha = weights(3, 512, 512, False)
    x = rows(T, 512, torch.bfloat16)
    _in_two_graphs(lambda: X.nvfp4_weight_product(x, codes[0], scales[0], alpha[:1]), [x])
    begin = torch.tensor([0, T // 2, T // 2, T], dtype=torch.int32, device="cuda")
    _in_two_graphs(lambda: X.nvfp4_experts_product(x, begin, codes, scales, alpha), [x])


def test_two_streams_at_once():
    """Nothing is shared between calls: many at once on two streams, of different sizes."""
    (codes, scales, alpha), xs = weights(4, 1024, 1024, True), [rows(T, 1024, torch.bfloat16, T) for T in (3, 700)]
    begin = [torch.tensor([0, 1, 1, 2, 3], dtype=torch.int32, device="cuda"), torch.tensor([0, 300, 301, 690, 700], dtype=torch.int32, device="cuda")]
    want = [X.nvfp4_experts_product(x, b, codes, scales, alpha, flags=B.GEMM_B_TILE_SCALES) for x, b in zip(xs, begin)]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(X.nvfp4_experts_product(xs[i], begin[i], codes, scales, alpha, flags=B.GEMM_B_TILE_SCALES, stream=s))
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        assert all(torch.equal(g, w) for g in got[i])


@pytest.mark.parametrize("T", [5, 200])
def test_linear_layer_of_a_weight_alone(T):
    """linear.fprop and dgrad with ``weight_only``: the library's products of the same operands, in the caller's types."""
    g = torch.Generator().manual_seed(1)
    q = L.quantize_weight(torch.randn((160, 96), generator=g).cuda())
    for x, dy in ((rows(T, 96, torch.bfloat16), rows(T, 160, torch.bfloat16, 3)), (rows(T, 96, torch.float32), rows(T, 160, torch.float32, 3))):
        w = values(q["codes_row"], q["scales_row"], True)
        ref = q["alpha"].double() * (x.double() @ w.T)
        close(L.fprop(x, q, weight_only=True), ref, bound(x, w, q["alpha"], ref, x.dtype, torch.bfloat16))
        ref = q["alpha"].double() * (dy.double() @ w)
        close(L.dgrad(dy, q, 0, weight_only=True), ref, bound(dy, w.T, q["alpha"], ref, dy.dtype, torch.bfloat16))


@pytest.mark.parametrize("T", [1, 40, 600])
@pytest.mark.parametrize("exponent", [-60, -110, -118, -126, -133, -140])
def test_the_least_numbers(T, exponent):
    """BF16 activations down to the least subnormal number are exact; of fp32 ones what lies below BF16's least number, 2^-133, is lost: less
    than that of each."""
    K, N = 96, 24
    codes, scales, alpha = weights(1, N, K, False)
    alpha = alpha * 0 + 2.0 ** 60
    w = values(codes[0], scales[0], False)
    for dtype, lost in ((torch.bfloat16, 0.0), (torch.float32, 2.0 ** -133)):
        x = (torch.rand((T, K), generator=torch.Generator().manual_seed(3)) * 2.0 ** exponent).to(dtype).cuda()
        ref = alpha.double() * (x.double() @ w.T)
        n = (3 if dtype == torch.float32 else 1) * K + 64
        off = float(alpha) * ((2 * n * U * x.double().abs() + lost) @ w.abs().T) + 2 * U * ref.abs()
        close(X.nvfp4_weight_product(x, codes[0], scales[0], alpha, out_dtype=B.OUT_F32), ref, off + U * ref.abs() + 2.0 ** -149)

"""Timed operators: serving and differentiating layers whose frozen weights are NVFP4, one projection or many experts.

  product           activations as they are (BF16 or fp32) times a weight of 4-bit codes with a scale of 16 each: y = x W^T
  experts           the same with a weight for each expert, for rows that stand in the order of their experts
  dispatch          tokens sorted by expert, and every token's row brought to its experts' places
  dispatch_backward the gradient of the rows brought there: of every token the sum over its places
  combine           the experts' rows back in the tokens' order, weighted and added up, on top of what is there
  combine_backward  the gradients of the same: of the experts' rows and of the weights

The plain forms are products, sums, comparisons and indexing in 32 bits, rounded once at the end.
"""
import functools
import math

import torch

own = False


def listed():
    return [
        # one new token through one projection: nothing but latency
        dict(name="product_1_4096x4096", kind="product", tokens=1, inp=4096, out=4096, tiles=False, dtype="bf16", result="bf16"),
        # a decoding batch, the weight packed in 16x16 tiles as it is where its transpose is needed too
        dict(name="product_24_8192x8192", kind="product", tokens=24, inp=8192, out=8192, tiles=True, dtype="bf16", result="bf16"),
        # a short prefill whose activations are still in fp32, as is its result; a vocabulary's odd number of columns
        dict(name="product_500_4096x10001_f32", kind="product", tokens=500, inp=4096, out=10001, tiles=False, dtype="f32",
             result="f32"),
        # the input's gradient in a training batch, through the packing of the transposed weight
        dict(name="product_4096_8192x8192", kind="product", tokens=4096, inp=8192, out=8192, tiles=True, dtype="bf16",
             result="bf16"),
        # a decoding batch through many small experts, few tokens each, some experts with none
        dict(name="experts_32_of_64", kind="experts", tokens=32, top=4, experts=64, inp=2048, out=1024, none=0.0, gather=True,
             tiles=False, dtype="bf16", result="bf16"),
        # a prefill through larger ones: hundreds of tokens for each, unevenly
        dict(name="experts_4096_of_32", kind="experts", tokens=4096, top=4, experts=32, inp=2048, out=4096, none=0.02, gather=True,
             tiles=False, dtype="bf16", result="bf16"),
        # the gradient through a few large experts, rows in the experts' order already, transposed packings
        dict(name="experts_1999_of_8_back", kind="experts", tokens=1999, top=2, experts=8, inp=4096, out=2880, none=0.1,
             gather=False, tiles=True, dtype="bf16", result="bf16"),
        # a decoding batch on its way to the experts
        dict(name="dispatch_64x4096", kind="dispatch", tokens=64, top=4, experts=64, width=4096, none=0.0, dtype="bf16"),
        # a training batch on its way there, padding among it
        dict(name="dispatch_16384x4096", kind="dispatch", tokens=16384, top=4, experts=64, width=4096, none=0.05, dtype="bf16"),
        # ... and its gradient on the way back, fp32 sums of fp32 rows
        dict(name="dispatch_backward_5001x2880_f32", kind="dispatch_backward", tokens=5001, top=6, experts=128, width=2880,
             none=0.05, dtype="f32"),
        # the experts' rows back, on top of what the layer's input left
        dict(name="combine_16384x4096", kind="combine", tokens=16384, top=4, experts=64, width=4096, none=0.05, dtype="bf16"),
        # the gradients of the same, a ragged batch
        dict(name="combine_backward_5001x2880", kind="combine_backward", tokens=5001, top=8, experts=128, width=2880, none=0.05,
             dtype="bf16"),
    ]


def _log_size(rng, lo, hi, multiple=1):
    """A multiple of `multiple` in [lo, hi], spread evenly over the logarithm."""
    v = lo * (hi / lo) ** rng.random()
    return max(lo, int(v) // multiple * multiple)


def draw(rng):
    kind = rng.choice(["product", "product", "product", "experts", "experts", "experts", "dispatch", "dispatch",
                       "dispatch_backward", "combine", "combine_backward"])
    if kind == "product":
        tiles = rng.random() < 0.4
        return dict(kind=kind, tokens=_log_size(rng, 1, 4096), inp=_log_size(rng, 32, 8192, 32),
                    out=_log_size(rng, 16, 8192, 16) if tiles else _log_size(rng, 1, 8192), tiles=tiles,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), result=rng.choice(["bf16", "bf16", "f32"]))
    experts = _log_size(rng, 1, 128)
    top = min(experts, rng.choice([1, 2, 2, 4, 4, 6, 8]))
    none = rng.choice([0.0, 0.02, 0.3])
    if kind == "experts":
        tiles = rng.random() < 0.4
        case = dict(kind=kind, tokens=_log_size(rng, 1, 4096), top=top, experts=experts, inp=_log_size(rng, 32, 4096, 32),
                    out=_log_size(rng, 16, 4096, 16) if tiles else _log_size(rng, 1, 4096), none=none, gather=rng.random() < 0.6,
                    tiles=tiles, dtype=rng.choice(["bf16", "bf16", "f32"]), result=rng.choice(["bf16", "bf16", "f32"]))
        while experts * case["inp"] * case["out"] > 1 << 28:               # no more weights than the largest listed one
            case["inp"] = max(32, case["inp"] // 64 * 32)
    else:
        case = dict(kind=kind, tokens=_log_size(rng, 1, 8192), top=top, experts=experts, width=_log_size(rng, 8, 8192, 8), none=none,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    while work(case)["flops"] > 3e11 or work(case)["bytes"] > 6e8:         # ... and no more to do
        case["tokens"] //= 2
    return case


# ---- inputs ------------------------------------------------------------------------------

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _quantized(E, N, K, tiles, g):
    """Weights of E experts [N][K], normal with a few larger columns, rounded to NVFP4: codes [E][N][K/2], scales of 16 each (or of
    16x16 tiles), alpha [E]."""
    codes = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((E, N // 16 if tiles else N, K // 16), dtype=torch.uint8, device="cuda")
    alpha = torch.empty(E, device="cuda")
    border = torch.tensor([(a + b) / 2 for a, b in zip(_GRID, _GRID[1:])], device="cuda")
    for e in range(E):
        w = torch.randn((N, K), generator=g, device="cuda") / math.sqrt(K)
        w *= torch.exp(0.5 * torch.randn(K, generator=g, device="cuda"))
        alpha[e] = w.abs().amax() / (6 * 448)
        blocks = w.view(N // 16, 16, K // 16, 16).abs().amax((1, 3)) if tiles else w.view(N, K // 16, 16).abs().amax(2)
        s = (blocks / (6 * alpha[e])).to(torch.float8_e4m3fn)
        scales[e] = s.view(torch.uint8)
        step = (s.float() * alpha[e]).repeat_interleave(16, 1)
        step = step.repeat_interleave(16, 0) if tiles else step
        y = torch.where(step > 0, w / step, 0)
        c = torch.bucketize(y.abs(), border).to(torch.uint8) | ((w < 0).to(torch.uint8) << 3)
        codes[e] = c[:, 0::2] | (c[:, 1::2] << 4)
    return codes, scales, alpha


def _ids(case, g):
    """The experts of every token, the most likely ones of an uneven router; -1 throughout for padding."""
    T, E, k = case["tokens"], case["experts"], case["top"]
    logits = 0.5 * torch.randn(E, generator=g, device="cuda") + torch.randn((T, E), generator=g, device="cuda")
    values, ids = logits.topk(k, dim=1)
    none = torch.rand(T, generator=g, device="cuda") < case["none"]
    return torch.where(none[:, None], -1, ids).to(torch.int32), torch.softmax(values, 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def rows(n, width, dtype):
        # of uneven magnitude, as activations are
        return (torch.randn((n, width), generator=g, device="cuda") * torch.exp(0.5 * torch.randn((n, 1), generator=g, device="cuda"))).to(
            _type(dtype))

    s = dict(kind=case["kind"], tiles=case.get("tiles", False), result=case.get("result", "bf16"))
    if case["kind"] == "product":
        s["x"] = rows(case["tokens"], case["inp"], case["dtype"])
        codes, scales, s["alpha"] = _quantized(1, case["out"], case["inp"], case["tiles"], g)
        s.update(codes=codes[0], scales=scales[0])
        return s
    T, k, E = case["tokens"], case["top"], case["experts"]
    ids, weights = _ids(case, g)
    s.update(ids=ids, experts=E)
    if case["kind"] == "dispatch":
        s["x"] = rows(T, case["width"], case["dtype"])
        return s
    place, token, begin = _sorted(ids, E)
    if case["kind"] == "experts":
        s.update(begin=begin, token=token if case["gather"] else None)
        s["x"] = rows(T if case["gather"] else T * k, case["inp"], case["dtype"])
        s["codes"], s["scales"], s["alpha"] = _quantized(E, case["out"], case["inp"], case["tiles"], g)
        return s
    s.update(place=place)
    slots = rows(T * k, case["width"], case["dtype"])
    if case["kind"] == "dispatch_backward":
        s["dxs"] = slots
        return s
    s.update(ys=slots, weights=weights)
    s["base" if case["kind"] == "combine" else "dy"] = rows(T, case["width"], case["dtype"])
    return s


# ---- one pass ----------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _package():
    from paper_2512_02010_amd import binding, experts
    return binding, experts


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    B, X = _package()
    kind = s["kind"]
    kw = dict(out_dtype=B.OUT_F32 if s["result"] == "f32" else B.OUT_BF16, flags=B.GEMM_B_TILE_SCALES if s["tiles"] else 0)
    if kind == "product":
        return dict(y=X.nvfp4_weight_product(s["x"], s["codes"], s["scales"], s["alpha"], **kw))
    if kind == "experts":
        return dict(ys=X.nvfp4_experts_product(s["x"], s["begin"], s["codes"], s["scales"], s["alpha"], token=s["token"], **kw))
    if kind == "dispatch":
        place, token, begin = X.nvfp4_experts_sort(s["ids"], s["experts"])
        return dict(xs=X.nvfp4_experts_spread(s["x"], place), place=place, token=token, begin=begin)
    if kind == "dispatch_backward":
        return dict(dx=X.nvfp4_experts_combine(s["dxs"], s["place"]))
    if kind == "combine":
        return dict(y=X.nvfp4_experts_combine(s["ys"], s["place"], s["weights"], base=s["base"]))
    dys, dw = X.nvfp4_experts_combine_backward(s["dy"], s["ys"], s["place"], s["weights"])
    return dict(dys=dys, dw=dw)


def _expanded(codes, scales, tiles):
    """codes times scales, fp32 (exact; without alpha)."""
    grid = torch.tensor(_GRID + tuple(-v for v in _GRID), device=codes.device)
    values = torch.stack((grid[(codes & 15).long()], grid[(codes >> 4).long()]), dim=2).flatten(1)
    s = scales.view(torch.float8_e4m3fn).float().repeat_interleave(16, 1)
    return values * (s.repeat_interleave(16, 0) if tiles else s)


def _sorted(ids, E):
    """place [T][k]: where the pair (token, j) stands in the order of the experts, ~place for one without an expert; token [T * k]
    of every such place (-1: no expert's); begin [E + 1] of every expert's places."""
    k = ids.shape[1]
    key = torch.where((ids >= 0) & (ids < E), ids, E).flatten()
    order = torch.argsort(key, stable=True)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(len(order), device=ids.device)
    begin = (key[:, None] < torch.arange(E + 1, device=ids.device)).sum(0)
    token = torch.where(key[order] < E, order // k, -1)
    return torch.where(key < E, slot, ~slot).reshape(ids.shape).to(torch.int32), token.to(torch.int32), begin.to(torch.int32)


def _run_plain(s):
    kind = s["kind"]
    if kind == "product":
        y = s["x"].float() @ _expanded(s["codes"], s["scales"], s["tiles"]).T * s["alpha"]
        return dict(y=y.to(_type(s["result"])))
    if kind == "experts":
        begin, x = s["begin"].tolist(), s["x"]
        S = len(x) if s["token"] is None else len(s["token"])
        ys = torch.zeros((S, s["codes"].shape[1]), dtype=_type(s["result"]), device="cuda")
        for e, (first, last) in enumerate(zip(begin, begin[1:])):
            if first < last:
                mine = x[first:last] if s["token"] is None else x[s["token"][first:last].long()]
                y = mine.float() @ _expanded(s["codes"][e], s["scales"][e], s["tiles"]).T
                ys[first:last] = (y * s["alpha"][e]).to(ys.dtype)
        return dict(ys=ys)
    if kind == "dispatch":
        place, token, begin = _sorted(s["ids"], s["experts"])
        xs = s["x"].float()[token.clamp(min=0).long()] * (token >= 0)[:, None]
        return dict(xs=xs.to(s["x"].dtype), place=place, token=token, begin=begin)
    there = s["place"] >= 0
    slot = torch.where(there, s["place"], ~s["place"]).long()
    if kind == "dispatch_backward":
        return dict(dx=_weighted(s["dxs"], slot, there.float()).to(s["dxs"].dtype))
    if kind == "combine":
        return dict(y=(s["base"].float() + _weighted(s["ys"], slot, s["weights"] * there)).to(s["base"].dtype))
    dy, weights = s["dy"].float(), s["weights"] * there
    dys = torch.zeros(s["ys"].shape, device="cuda")
    dw = torch.empty_like(weights)
    for j in range(slot.shape[1]):
        dys[slot[:, j]] = weights[:, j, None] * dy
        dw[:, j] = (dy * s["ys"][slot[:, j]].float()).sum(1) * there[:, j]
    return dict(dys=dys.to(s["ys"].dtype), dw=dw)


def _weighted(ys, slot, weights):
    total = torch.zeros((len(slot), ys.shape[1]), device=ys.device)
    for j in range(slot.shape[1]):
        total += weights[:, j, None] * ys[slot[:, j]].float()
    return total


# ---- what a pass cannot do without -------------------------------------------------------------

def work(case):
    size = 4 if case.get("dtype") == "f32" else 2
    T = case["tokens"]
    if case["kind"] in ("product", "experts"):
        K, N = case["inp"], case["out"]
        weight = N * K // 2 + (N // 16 if case["tiles"] else N) * (K // 16)
        result = 4 if case["result"] == "f32" else 2
        if case["kind"] == "product":
            return dict(bytes=size * T * K + weight + result * T * N, flops=2 * T * N * K)
        S, E = T * case["top"], case["experts"]
        learnt = S * (1 - case["none"])
        used = E * (1 - (1 - 1 / E) ** learnt) if E > 1 else 1             # experts that some token has, were they all as likely
        return dict(bytes=size * K * (T if case["gather"] else S) + used * weight + result * S * N + 4 * S + 4 * E,
                    flops=2 * learnt * N * K)
    S, W = T * case["top"], case["width"]
    there = S * (1 - case["none"])
    if case["kind"] == "dispatch":
        return dict(bytes=size * W * (T + S) + 12 * S, flops=0)
    if case["kind"] == "dispatch_backward":
        return dict(bytes=size * W * (T + there) + 4 * S, flops=W * there)
    if case["kind"] == "combine":
        return dict(bytes=size * W * (2 * T + there) + 8 * S, flops=2 * W * there)
    return dict(bytes=size * W * (T + there + S) + 12 * S, flops=3 * W * there)


# ---- the operators' definitions in 64 bits -----------------------------------------------------

def _value(codes, scales):
    """[N][K] from codes [N][K/2] and one scale byte for each of 16: sign, exponent and mantissa spelled out."""
    nibbles = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.int64, device=codes.device)
    nibbles[:, 0::2], nibbles[:, 1::2] = codes & 0xF, codes >> 4
    exponent, half = nibbles >> 1 & 3, (nibbles & 1).double()
    magnitude = torch.where(exponent == 0, half / 2, (1 + half / 2) * 2.0 ** (exponent - 1).double())
    byte = scales.long()
    e, m = byte >> 3, (byte & 7).double()
    scale = torch.where(e == 0, m / 512, (1 + m / 8) * 2.0 ** (e - 7).double())
    return torch.where(nibbles >= 8, -magnitude, magnitude) * scale[:, torch.arange(nibbles.shape[1], device=codes.device) // 16]


def _weight(s, e=None):
    codes, scales = (s["codes"], s["scales"]) if e is None else (s["codes"][e], s["scales"][e])
    if s["tiles"]:
        scales = scales[torch.arange(len(codes), device="cuda") // 16]
    return _value(codes, scales) * s["alpha"][e or 0].double()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "product":
        return dict(y=s["x"].double() @ _weight(s).T)
    E, ids = case["experts"], s["ids"]
    flat = ids.flatten().long()
    T, k = ids.shape
    # places by counting: an expert's pairs stand behind those of lower experts and behind its own of lower number
    which = torch.where((flat < 0) | (flat >= E), E, flat)
    hot = which[:, None] == torch.arange(E + 1, device="cuda")
    count = hot.sum(0)
    first = torch.cat((count.new_zeros(1), count.cumsum(0)))
    slot = (first[which] + hot.cumsum(0).gather(1, which[:, None])[:, 0] - 1).reshape(T, k)
    kept = (which < E).reshape(T, k)
    token = torch.full((T * k,), -1, dtype=torch.int64, device="cuda")
    pairs = torch.arange(T, device="cuda")[:, None].expand(T, k)
    token[slot[kept]] = pairs[kept]
    if kind == "experts":
        ys = torch.zeros((T * k, case["out"]), dtype=torch.float64, device="cuda")
        x = s["x"].double()
        for e in range(E):
            mine = torch.arange(int(first[e]), int(first[e + 1]), device="cuda")
            if len(mine):
                ys[mine] = x[token[mine] if case["gather"] else mine] @ _weight(s, e).T
        return dict(ys=ys)
    if kind == "dispatch":
        xs = torch.zeros((T * k, case["width"]), dtype=torch.float64, device="cuda")
        xs[slot[kept]] = s["x"].double()[pairs[kept]]
        return dict(xs=xs, place=torch.where(kept, slot, -1 - slot).int(), token=token.int(), begin=first[: E + 1].int())
    total = torch.zeros((T, case["width"]), dtype=torch.float64, device="cuda")
    if kind in ("dispatch_backward", "combine"):
        if kind == "combine":
            total += s["base"].double()
        for j in range(k):
            mine = kept[:, j]
            part = s["dxs" if kind == "dispatch_backward" else "ys"][slot[mine, j]].double()
            total[mine] += part if kind == "dispatch_backward" else part * s["weights"][mine, j, None].double()
        return dict(dx=total) if kind == "dispatch_backward" else dict(y=total)
    dys = torch.zeros((T * k, case["width"]), dtype=torch.float64, device="cuda")
    dw = torch.zeros((T, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        mine = kept[:, j]
        dy = s["dy"][mine].double()
        dys[slot[mine, j]] = s["weights"][mine, j, None].double() * dy
        dw[mine, j] = (dy * s["ys"][slot[mine, j]].double()).sum(1)
    return dict(dys=dys, dw=dw)

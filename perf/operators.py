"""Timed operators: what recovers, and then serves, a model whose weights are quantized to NVFP4.

  adapters_forward    low-rank adapters of many requests at once beside a shared projection: every token has
                      an adapter of its own, or none, and the projection's output comes out with it added
  adapters_backward   the gradients of the same: of the tokens and of every adapter
  distill_forward     the divergence of a model's logits from a teacher's top logits, one loss per token
  distill_backward    its gradient for the logits, from what the forward pass kept
  distill_step        both in one call, as a training step without a graph between them makes it

The plain forms are products, sums, exponentials and indexing in 32 bits, rounded once at the end.
"""
import functools
import math

import torch

own = False


def listed():
    return [
        # one new token of one request: nothing but latency
        dict(name="decode_1_4096x4096", kind="adapters_forward", tokens=1, inp=4096, out=4096, rank=16, adapters=4,
             order="mixed", none=0.0, keep=False, dtype="bf16"),
        # a decoding batch: one token of each request, adapters in any order, some requests without one
        dict(name="decode_64_8192x8192", kind="adapters_forward", tokens=64, inp=8192, out=8192, rank=16, adapters=32,
             order="mixed", none=0.15, keep=False, dtype="bf16"),
        # a short, ragged prefill of several requests, the projection's output still in fp32
        dict(name="prefill_1000_4096x4096", kind="adapters_forward", tokens=1000, inp=4096, out=4096, rank=64, adapters=8,
             order="segments", none=0.1, keep=False, dtype="f32"),
        # the forward pass of a training batch, the low-rank activations kept for the backward pass
        dict(name="train_16384_4096x4096", kind="adapters_forward", tokens=16384, inp=4096, out=4096, rank=16, adapters=4,
             order="segments", none=0.0, keep=True, dtype="bf16"),
        # the backward pass of a step with one adapter
        dict(name="grad_2048_4096x4096", kind="adapters_backward", tokens=2048, inp=4096, out=4096, rank=16, adapters=1,
             order="segments", none=0.0),
        # ... and of a large step that trains several, sequences of which are packed one after the other
        dict(name="grad_8192_8192x8192", kind="adapters_backward", tokens=8192, inp=8192, out=8192, rank=32, adapters=8,
             order="segments", none=0.05),
        # a few tokens of an evaluation, small vocabulary
        dict(name="loss_7x32000", kind="distill_forward", tokens=7, vocab=32000, top=16, temperature=1.0, dtype="bf16"),
        # a batch whose vocabulary is odd, so that no two rows begin alike
        dict(name="loss_4096x50021", kind="distill_forward", tokens=4096, vocab=50021, top=64, temperature=2.0, dtype="bf16"),
        # gradients of fp32 logits
        dict(name="dlogits_1024x32768_f32", kind="distill_backward", tokens=1024, vocab=32768, top=32, temperature=1.0,
             dtype="f32"),
        # ... and of a ragged batch in BF16
        dict(name="dlogits_2047x50021", kind="distill_backward", tokens=2047, vocab=50021, top=100, temperature=2.0,
             dtype="bf16"),
        # a small step in fp32
        dict(name="step_255x50021_f32", kind="distill_step", tokens=255, vocab=50021, top=100, temperature=1.5, dtype="f32"),
        # a training step over a large vocabulary
        dict(name="step_4096x131072", kind="distill_step", tokens=4096, vocab=131072, top=64, temperature=1.0, dtype="bf16"),
    ]


def _log_size(rng, lo, hi, multiple=1):
    """A multiple of `multiple` in [lo, hi], spread evenly over the logarithm."""
    v = lo * (hi / lo) ** rng.random()
    return max(lo, int(v) // multiple * multiple)


def draw(rng):
    kind = rng.choice(["adapters_forward", "adapters_forward", "adapters_backward", "adapters_backward", "distill_forward",
                       "distill_backward", "distill_step"])
    if kind.startswith("adapters"):
        case = dict(kind=kind, tokens=_log_size(rng, 1, 8192), inp=_log_size(rng, 64, 8192, 8), out=_log_size(rng, 64, 8192, 8),
                    rank=rng.choice([1, 4, 8, 8, 12, 16, 16, 16, 32, 32, 64, 100, 128]), adapters=_log_size(rng, 1, 64),
                    order=rng.choice(["segments", "mixed"]), none=rng.choice([0.0, 0.1, 0.5]))
        case["adapters"] = min(case["adapters"], max(1, 1024 // case["rank"]))
        if kind == "adapters_forward":
            case.update(keep=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]))
        return case
    return dict(kind=kind, tokens=_log_size(rng, 1, 4096), vocab=_log_size(rng, 1000, 65536), top=_log_size(rng, 1, 256),
                temperature=rng.choice([0.7, 1.0, 2.0]), dtype=rng.choice(["bf16", "bf16", "f32"]))


# ---- inputs ------------------------------------------------------------------------------

def _type(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _which(case, g):
    """The adapter of every token: requests one after the other, or in any order; -1 for none."""
    T, L = case["tokens"], case["adapters"]
    if case["order"] == "mixed":
        which = torch.randint(0, L, (T,), generator=g, device="cuda")
        none = torch.rand(T, generator=g, device="cuda") < case["none"]
    else:
        requests = max(1, min(T, 2 * L))
        cuts = torch.rand(T, generator=g, device="cuda").argsort()[: requests - 1]
        begins = torch.zeros(T, dtype=torch.int64, device="cuda")
        begins[cuts] = 1
        request = begins.cumsum(0) % requests
        which = torch.randint(0, L, (requests,), generator=g, device="cuda")[request]
        none = (torch.rand(requests, generator=g, device="cuda") < case["none"])[request]
    return torch.where(none, -1, which).to(torch.int32)


def _adapters_state(case, g):
    T, K, N, r, L = (case[k] for k in ("tokens", "inp", "out", "rank", "adapters"))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    # tokens of uneven magnitude, as the layers' activations are; adapters of a size that the projection's own output has too
    s = dict(x=(normal(T, K) * torch.exp(0.5 * normal(T, 1))).bfloat16(), a=(normal(L, r, K) / math.sqrt(K)).bfloat16(),
             b=(normal(L, N, r) / math.sqrt(r)).bfloat16(), which=_which(case, g),
             scales=0.5 + torch.rand(L, generator=g, device="cuda"))
    if case["kind"] == "adapters_forward":
        s["base"] = normal(T, N).to(_type(case))
    else:
        s["dy"] = (1e-3 * normal(T, N) * torch.exp(normal(T, 1))).bfloat16()
        s["dx_base"] = (1e-3 * normal(T, K)).bfloat16()
        s["h"] = _low_rank(s["x"].float(), s["a"].float(), s["which"])
    return s


def _distill_state(case, g):
    T, V, k = case["tokens"], case["vocab"], min(case["top"], case["vocab"])
    rows = max(1, (1 << 27) // V)
    logits = torch.empty((T, V), dtype=_type(case), device="cuda")
    teacher = torch.empty((T, k), dtype=torch.float32, device="cuda")
    index = torch.empty((T, k), dtype=torch.int32, device="cuda")
    for t in range(0, T, rows):                     # (a part at a time: fp32 copies of the largest would fill the memory)
        z = 2.5 * torch.randn((min(rows, T - t), V), generator=g, device="cuda")
        logits[t:t + rows] = z
        z += 0.7 * torch.randn(z.shape, generator=g, device="cuda")
        teacher[t:t + rows], top = z.topk(k, dim=1)
        index[t:t + rows] = top.to(torch.int32)
    # lists that end early, and tokens that are not learnt from (prompts, padding): no list at all
    length = torch.randint((k + 1) // 2, k + 1, (T, 1), generator=g, device="cuda")
    skipped = torch.rand((T, 1), generator=g, device="cuda") < (0.1 if T > 1 else 0.0)
    length = torch.where(skipped, 0, length)
    index[torch.arange(k, device="cuda")[None] >= length] = -1
    s = dict(logits=logits, teacher=teacher, index=index, temperature=float(case["temperature"]))
    if case["kind"] != "distill_forward":
        s["weight"] = (0.5 + torch.rand(T, generator=g, device="cuda")) / T
    if case["kind"] == "distill_backward":
        s["lse"] = torch.empty(T, device="cuda")
        for t in range(0, T, rows):
            s["lse"][t:t + rows] = _lse(logits[t:t + rows].float() * (1 / s["temperature"]))
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = (_adapters_state if case["kind"].startswith("adapters") else _distill_state)(case, g)
    s.update(kind=case["kind"], keep=case.get("keep", False))
    return s


# ---- one pass ----------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _package():
    from paper_2512_02010_amd import finetune
    return finetune


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    F, kind = _package(), s["kind"]
    if kind == "adapters_forward":
        got = F.nvfp4_adapters_forward(s["x"], s["base"], s["a"], s["b"], s["which"], s["scales"], want_h=s["keep"])
        return dict(out=got[0], h=got[1]) if s["keep"] else dict(out=got)
    if kind == "adapters_backward":
        dx, da, db = F.nvfp4_adapters_backward(s["dy"], s["x"], s["h"], s["a"], s["b"], s["which"], s["scales"], s["dx_base"])
        return dict(dx=dx, da=da, db=db)
    if kind == "distill_forward":
        loss, lse = F.nvfp4_distill_forward(s["logits"], s["teacher"], s["index"], s["temperature"])
        return dict(loss=loss, lse=lse)
    if kind == "distill_backward":
        return dict(dlogits=F.nvfp4_distill_backward(s["logits"], s["teacher"], s["index"], s["lse"], s["weight"],
                                                     s["temperature"]))
    loss, dlogits = F.nvfp4_distill_step(s["logits"], s["teacher"], s["index"], s["weight"], s["temperature"])
    return dict(loss=loss, dlogits=dlogits)


def _low_rank(x, a, which):
    """h [T][r]: every token times the matrix A of its own adapter; 0 without one."""
    L, r, K = a.shape
    every = (x @ a.reshape(L * r, K).T).reshape(-1, L, r)
    h = every[torch.arange(len(which), device=which.device), which.clamp(min=0).long()]
    return torch.where(which[:, None] >= 0, h, 0)


def _placed(h, which, scales):
    """[T][L * r]: scale * h in the columns of the token's adapter, 0 in the others."""
    L = len(scales)
    mine = which[:, None] == torch.arange(L, device=which.device, dtype=which.dtype)
    return ((mine * scales)[:, :, None] * h[:, None, :]).reshape(len(which), -1)


def _run_plain(s):
    if s["kind"] == "adapters_forward":
        a, b = s["a"].float(), s["b"].float()
        h = _low_rank(s["x"].float(), a, s["which"])
        out = s["base"].float() + _placed(h, s["which"], s["scales"]) @ b.transpose(1, 2).reshape(-1, b.shape[1])
        out = out.to(s["base"].dtype)
        return dict(out=out, h=h) if s["keep"] else dict(out=out)
    if s["kind"] == "adapters_backward":
        (L, r, K), N = s["a"].shape, s["b"].shape[1]
        x, dy, a, bt = s["x"].float(), s["dy"].float(), s["a"].float(), s["b"].float().transpose(1, 2)
        dh = _placed(_low_rank(dy, bt, s["which"]), s["which"], s["scales"])
        dx = s["dx_base"].float() + dh @ a.reshape(L * r, K)
        db = dy.T @ _placed(s["h"], s["which"], s["scales"])
        return dict(dx=dx.bfloat16(), da=(dh.T @ x).reshape(L, r, K), db=db.reshape(N, L, r).transpose(0, 1).contiguous())
    y = s["logits"].float() * (1 / s["temperature"])
    p, rest, at = _target(s)
    learnt = p.sum(1) > 0
    if s["kind"] == "distill_backward":
        lse = s["lse"]
    else:
        lse = _lse(y)
        loss = torch.where(p > 0, p * (rest - (y.gather(1, at) - lse[:, None])), 0).sum(1)
        if s["kind"] == "distill_forward":
            return dict(loss=loss, lse=lse)
    d = torch.where(learnt[:, None], torch.exp(y - lse[:, None]), 0)
    d = (d.scatter_add(1, at, -p) * (s["weight"] / s["temperature"])[:, None]).to(s["logits"].dtype)
    return dict(dlogits=d) if s["kind"] == "distill_backward" else dict(loss=loss, dlogits=d)


def _lse(y):
    m = y.amax(1)
    return m + torch.log(torch.exp(y - m[:, None]).sum(1))


def _target(s):
    """The teacher's distribution over its list, its logarithm, and the places of the list (0 for what is no entry)."""
    listed_ = s["index"] >= 0
    t = torch.where(listed_, s["teacher"] * (1 / s["temperature"]), -torch.inf)
    m = torch.where(listed_.any(1), t.amax(1), 0)
    e = torch.exp(t - m[:, None])
    total = e.sum(1).clamp(min=torch.finfo(torch.float32).tiny)
    return e / total[:, None], t - m[:, None] - torch.log(total)[:, None], s["index"].clamp(min=0).long()


# ---- what a pass cannot do without -------------------------------------------------------------

def work(case):
    size = 4 if case.get("dtype") == "f32" else 2
    if case["kind"].startswith("adapters"):
        T, K, N, r, L = (case[k] for k in ("tokens", "inp", "out", "rank", "adapters"))
        learnt, used = T * (1 - case["none"]), min(L, T)
        weights = used * r * (K + N)
        if case["kind"] == "adapters_forward":
            return dict(bytes=2 * T * K + 2 * size * T * N + 2 * weights + 4 * T + 4 * L + (4 * T * r if case["keep"] else 0),
                        flops=2 * learnt * r * (K + N))
        return dict(bytes=2 * T * N + 6 * T * K + 4 * T * r + 2 * weights + 4 * L * r * (K + N) + 4 * T + 4 * L,
                    flops=4 * learnt * r * (K + N))
    T, V, k = case["tokens"], case["vocab"], min(case["top"], case["vocab"])
    lists = 8 * T * k
    if case["kind"] == "distill_forward":
        return dict(bytes=size * T * V + lists + 8 * T, flops=4 * T * V)
    if case["kind"] == "distill_backward":
        return dict(bytes=2 * size * T * V + lists + 8 * T, flops=4 * T * V)
    return dict(bytes=2 * size * T * V + lists + 8 * T, flops=8 * T * V)


# ---- the operators' definitions in 64 bits -----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("adapters"):
        return _exact_adapters(case, s)
    T, V, k = case["tokens"], case["vocab"], s["index"].shape[1]
    tau, part = float(case["temperature"]), max(1, (1 << 27) // V)
    loss = torch.zeros(T, dtype=torch.float64, device="cuda")
    lse = torch.zeros(T, dtype=torch.float64, device="cuda")
    back = case["kind"] != "distill_forward"
    d = torch.zeros((T, V), dtype=torch.float64, device="cuda") if back else None
    for t in range(0, T, part):
        z = s["logits"][t:t + part].double() / tau
        top, at = s["teacher"][t:t + part].double() / tau, s["index"][t:t + part].long()
        lse[t:t + part] = torch.logsumexp(z, 1)
        if case["kind"] == "distill_backward":
            lse[t:t + part] = s["lse"][t:t + part].double()
        valid = at >= 0
        log_p = torch.log_softmax(top.masked_fill(~valid, -1e300), 1)
        p = torch.where(valid, log_p.exp(), 0.0)
        log_q = z - lse[t:t + part, None]
        loss[t:t + part] = torch.where(valid, p * (log_p - log_q.gather(1, at.clamp(min=0))), 0.0).sum(1)
        if back:
            part_d = d[t:t + part]
            part_d.copy_(log_q.exp_() * valid.any(1, keepdim=True))
            rows = torch.arange(len(part_d), device="cuda")[:, None].expand(-1, k)
            part_d.index_put_((rows[valid], at[valid]), -p[valid], accumulate=True)
            part_d.mul_(s["weight"][t:t + part, None].double() / tau)
    if case["kind"] == "distill_forward":
        return dict(loss=loss, lse=lse)
    return dict(dlogits=d) if case["kind"] == "distill_backward" else dict(loss=loss, dlogits=d)


def _exact_adapters(case, s):
    x, a, b, scales = (s[k].double() for k in ("x", "a", "b", "scales"))
    which = s["which"]
    if case["kind"] == "adapters_forward":
        out, h = s["base"].double(), torch.zeros((len(x), a.shape[1]), dtype=torch.float64, device="cuda")
        for i in range(len(a)):
            mine = (which == i).nonzero()[:, 0]
            h[mine] = x[mine] @ a[i].T
            out[mine] += scales[i] * (h[mine] @ b[i].T)
        return dict(out=out, h=h) if case["keep"] else dict(out=out)
    dy, h, dx = s["dy"].double(), s["h"].double(), s["dx_base"].double()
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for i in range(len(a)):
        mine = (which == i).nonzero()[:, 0]
        dh = scales[i] * (dy[mine] @ b[i])
        dx[mine] += dh @ a[i]
        da[i] = dh.T @ x[mine]
        db[i] = scales[i] * (dy[mine].T @ h[mine])
    return dict(dx=dx, da=da, db=db)

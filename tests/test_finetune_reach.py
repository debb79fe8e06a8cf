"""CPU: the sizes that the GPU tests of adapters and distillation run reach every kernel that the library has for them, and
every loop that such a kernel has: more than one tile a workgroup, a change of adapter, more than one row."""
import re
import subprocess
from itertools import groupby

import numpy as np

from paper_2512_02010_amd import build

from . import _finetune_sizes as sizes
from . import _hip_calls
from .test_gpu_adapters import SIZES as ADAPTERS_SMALL
from .test_gpu_adapters import _which
from .test_gpu_distill import SIZES as DISTILL_SMALL

EVERY_ADAPTER = [s[:6] for s in ADAPTERS_SMALL + sizes.ADAPTERS + sizes.ADAPTERS_FEW]


def _kernels():
    """address in the library -> (kernel, its parameters)"""
    table = {}
    for line in subprocess.run(["nm", str(build.SO)], text=True, capture_output=True, check=True).stdout.splitlines():
        at, _, name = line.split(maxsplit=2) if len(line.split()) == 3 else ("0", "", "")
        m = re.search(r"\d(k_(?:plan|shrink|expand|outer|join|distill_\w+?))(?:I(\w+?)E+v|E)", name)
        if m and "__device_stub__" not in name and not name.endswith(".kd"):
            parameters = tuple({"DF16b": "bf16", "f": "f32"}.get(p, p.strip("LbiE")) for p in re.findall(r"L[bi]\d+E|DF16b|f", (m.group(2) or "") + "E"))
            table[int(at, 16)] = (m.group(1), parameters)
    return table


def _launches():
    """Of every call: its kernels and their grids' width."""
    adapters, distill = _hip_calls.run(f"""
from paper_2512_02010_amd import finetune as F
import subprocess
lib = F.lib()
at = C.cast(lib.nvfp4_distill_step, C.c_void_p).value
def kinds():
    return [(c[1] - at, c[3]) for c in calls() if c[0] == "launch"]
adapters = []
for T, K, N, r, L, _ in {EVERY_ADAPTER!r}:
    one = []
    for dtype in (0, 1):
        p = F.AdaptersParams(T, K, N, L, r, K, N, N, N, dtype)
        assert lib.nvfp4_adapters_forward(P, C.byref(p), P, P, P, P, P, P, P, P, 1 << 50, None) == 0
        one.append(kinds())
    p = F.AdaptersParams(T, K, N, L, r, K, K, K, N, 0)
    assert lib.nvfp4_adapters_backward(P, C.byref(p), P, P, P, P, P, P, P, P, P, P, P, 1 << 50, None) == 0
    one.append(kinds())
    adapters.append(one)
distill = []
for i, (T, V, k) in enumerate({DISTILL_SMALL + sizes.DISTILL!r}):
    one = []
    for dtype in (0, 1):
        v = V // 2 if dtype and i >= {len(DISTILL_SMALL)} else V
        d = F.DistillParams(T, v, v, k, 1.0, dtype, 1, 0)
        assert lib.nvfp4_distill_forward(P, C.byref(d), P, P, P, P, None) == 0
        assert lib.nvfp4_distill_backward(P, C.byref(d), P, P, P, P, P, None) == 0
        assert lib.nvfp4_distill_step(P, C.byref(d), P, P, P, P, P, None) == 0
        one.append(kinds())
    distill.append(one)
result = adapters, distill
""")
    out = subprocess.run(["nm", "-D", str(build.SO)], text=True, capture_output=True, check=True).stdout
    base = int(re.search(r"(\w+) T nvfp4_distill_step$", out, flags=re.M).group(1), 16)
    names = _kernels()

    def named(call):
        return [(*names[base + at], grid) for at, grid in call]

    return [[named(c) for c in one] for one in adapters], [[named(c) for c in one] for one in distill], set(names.values())


def _tiles(T, L, order, seed=1):
    """The adapters of the planned tiles (-1: none) and their tokens."""
    which = _which(T, L, order, seed).numpy()
    which = np.where((which >= 0) & (which < L), which, L)
    return [(a if a < L else -1, min(32, n - i)) for a, n in enumerate(np.bincount(which, minlength=L + 1)) for i in range(0, n, 32)]


def _stretches(units, workgroups):
    per = -(-len(units) // workgroups)
    return [units[i:i + per] for i in range(0, len(units), per)]


def _loops(units, workgroups):
    """What a kernel that deals `units` (adapters; None: an empty one) out goes through."""
    seen = set()
    for stretch in _stretches(units, workgroups):
        stretch = [a for a in stretch if a is not None and a >= 0]
        runs = [len(list(g)) for _, g in groupby(stretch)]
        if runs and max(runs) >= 3:
            seen.add("several tiles of an adapter")
        if len(runs) >= 2:
            seen.add("several adapters")
    return seen


def test_every_kernel_and_loop_is_reached():
    adapters, distill, known = _launches()
    launched = {(k, p) for calls in adapters + distill for call in calls for k, p, _ in call}
    assert launched == known, sorted(known - launched)

    seen = {}
    for (T, K, N, r, L, order), calls in zip(EVERY_ADAPTER, adapters):
        tiles = _tiles(T, L, order)
        halves = [a if n > 16 * h else None for a, n in tiles for h in (0, 1)]
        for call in calls:
            for kernel, parameters, grid in call:
                if kernel in ("k_shrink", "k_expand") and parameters[0] == "0":      # (not those for few tokens)
                    seen.setdefault((kernel, parameters), set()).update(
                        _loops(halves if kernel == "k_shrink" else [a for a, _ in tiles], grid))
        # k_outer: every fourth tile of an adapter within a range goes to one wave
        chunks = -(-K // 128) + -(-N // 128)
        most = T // 32 + min(L + 1, T)
        per = max(4, -(-most // -(-512 // chunks)))
        ranges = [list(g) for i in range(0, len(tiles), per) for _, g in groupby(a for a, _ in tiles[i:i + per] if a >= 0)]
        if T > 512:
            for kernel, parameters, _ in calls[2]:
                if kernel == "k_outer":
                    at = seen.setdefault((kernel, parameters), set())
                    if any(len(g) >= 9 for g in ranges):
                        at.add("several tiles of a wave")
                    if len(ranges) > len({a for a, _ in tiles if a >= 0}):
                        at.add("an adapter in several ranges")
    wanted = {"several tiles of an adapter", "several adapters"}
    missed = []
    for (kernel, parameters), loops in sorted(seen.items()):
        want = {"several tiles of a wave", "an adapter in several ranges"} if kernel == "k_outer" else wanted
        missed += [(kernel, parameters, what) for what in sorted(want - loops)]
    assert not missed, "\n".join(map(str, missed))

    rows = {}
    for (T, _, _), calls in zip(DISTILL_SMALL + sizes.DISTILL, distill):
        for call in calls:
            for kernel, parameters, grid in call:
                if kernel == "k_distill_rows":
                    rows[parameters] = max(rows.get(parameters, 0), T / grid)
    assert len(rows) == 30 and min(rows.values()) > 2, rows

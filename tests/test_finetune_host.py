"""CPU: what adapters and distillation ask of the HIP runtime (see _hip_calls.py), and the resources of their kernels."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

from paper_2512_02010_amd import build

from . import _hip_calls


def test_launches_of_a_call():
    """Adapters: two launches for few tokens, three with a plan; backwards five, four where an adapter's gradients are one
    workgroup's sums.  Distillation: one.  Nothing else is asked of the runtime."""
    counts = _hip_calls.run("""
from paper_2512_02010_amd import finetune as F
lib, result = F.lib(), {}
def kinds():
    return [c[0] for c in calls()]
for T in (1, 192, 193, 5000):
    for rank in (3, 16, 64, 100):
        for dtype in (0, 1):
            p = F.AdaptersParams(T, 512, 1024, 4, rank, 512, 1024, 1024, 1024, dtype)
            assert lib.nvfp4_adapters_forward(P, C.byref(p), P, P, P, P, P, P, P, P, 1 << 40, None) == 0
            result[f"forward {T} {rank} {dtype}"] = kinds()
for T in (0, 1, 512, 513, 5000):
    for rank in (3, 16, 64, 100):
        p = F.AdaptersParams(T, 512, 1024, 4, rank, 512, 512, 512, 1024, 0)
        assert lib.nvfp4_adapters_backward(P, C.byref(p), P, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == 0
        result[f"backward {T} {rank}"] = kinds()
for V in (1, 1000, 50000, 131072, 200000, 1 << 20):
    for dtype in (0, 1):
        d = F.DistillParams(300, V, V, 64, 1.0, dtype, 1, 0)
        assert lib.nvfp4_distill_forward(P, C.byref(d), P, P, P, P, None) == 0
        assert lib.nvfp4_distill_backward(P, C.byref(d), P, P, P, P, P, None) == 0
        assert lib.nvfp4_distill_step(P, C.byref(d), P, P, P, P, P, None) == 0
        result[f"distill {V} {dtype}"] = kinds()
""")
    for name, kinds in counts.items():
        what, n = name.split()[:2]
        want = {"forward": 2 if int(n) <= 192 else 3, "backward": 2 if n == "0" else 4 if int(n) <= 512 else 5, "distill": 3}[what]
        assert kinds == ["launch"] * want, (name, kinds)


def _report(source):
    flags = [f for f in build.HIPCC_FLAGS if f != "-shared"]
    r = subprocess.run([build.hipcc(), *flags, f"-I{build.ROOT / 'include'}", f"-I{build.PKG / 'csrc'}",
                        "-Rpass-analysis=kernel-resource-usage", "-c", str(build.PKG / "csrc" / source), "-o", "/dev/null"],
                       capture_output=True, text=True, check=True)
    kernels, cur = {}, None
    for line in r.stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            cur = kernels.setdefault(m.group(1), {})
            continue
        m = re.search(r"remark:\s+(VGPRs|ScratchSize \[bytes/lane\]|Occupancy \[waves/SIMD\]|LDS Size \[bytes/block\]): (\d+)", line)
        if m and cur is not None:
            cur[m.group(1).split(" ")[0]] = int(m.group(2))
    return kernels


def test_registers_of_the_streaming_kernels():
    """Columns of w, rows of logits and sums live in registers: none of these kernels may spill, and the small ranks leave
    room for two workgroups of k_shrink (four waves per SIMD), a row of k_distill_rows for the sixteen waves that it has."""
    with ThreadPoolExecutor(2) as pool:
        adapters, distill = pool.map(_report, ("adapters.hip", "distill.hip"))
    shrink = {k: v for k, v in adapters.items() if "k_shrink" in k}
    outer = {k: v for k, v in adapters.items() if "k_outer" in k}
    rows = {k: v for k, v in distill.items() if "k_distill_rows" in k}
    assert len(shrink) >= 20 and len(outer) == 3 and len(rows) == 30
    for name, v in {**shrink, **outer, **distill}.items():
        assert v["ScratchSize"] == 0, (name, v)
    for name, v in shrink.items():
        few, across, rt, nf = map(int, re.search(r"k_shrinkILb(\d)ELb(\d)ELi(\d)ELi(\d)E", name).groups())
        assert v["Occupancy"] >= (4 if rt <= 2 and rt * nf <= 8 else 2), (name, v)
    for name, v in rows.items():
        assert v["Occupancy"] >= 4, (name, v)

"""CPU: the sizes that the GPU tests of the products and of the routing run reach every kernel that the library has for them, by the calls' own
launches."""
import re
import subprocess

from paper_2512_02010_amd import build

from . import _hip_calls
from .test_gpu_experts import ROWS, ROWS_LARGE
from .test_gpu_weight_product import EXPERTS, SIZES

NAMES = r"k_few|k_tiles|k_sort|k_sort_count|k_spread|k_combine|k_combine_backward"


def _kernels():
    """address in the library -> kernel with its parameters"""
    table = {}
    for line in subprocess.run(["nm", str(build.SO)], text=True, capture_output=True, check=True).stdout.splitlines():
        at, _, name = line.split(maxsplit=2) if len(line.split()) == 3 else ("0", "", "")
        if re.search(rf"\d({NAMES})(I|E)", name) and "__device_stub__" not in name and not name.endswith(".kd"):
            table[int(at, 16)] = re.sub(r".*GLOBAL__N_1\d+", "", name)
    return table


def test_every_kernel_is_reached():
    launched = _hip_calls.run(f"""
from paper_2512_02010_amd import finetune as F
lib = F.lib()
at = C.cast(lib.nvfp4_distill_step, C.c_void_p).value
def take():
    return [c[1] - at for c in calls() if c[0] == "launch"]
result = []
for T, K, N, tiles in {SIZES!r}:
    for x in (0, 1):
        for out in (0, 1):
            p = F.ProductParams(T, K, N, 1, T, K, N, x, out, 2 if tiles else 0)
            assert lib.nvfp4_weight_product(P, C.byref(p), P, P, P, P, None) == 0
            result += take()
for T, k, E, K, N, tiles in {EXPERTS!r}:
    for x, out in ((0, 0), (0, 1), (1, 1), (1, 0)):
        p = F.ProductParams(T, K, N, E, T * k, K, N, x, out, 2 if tiles else 0)
        assert lib.nvfp4_experts_product(P, C.byref(p), P, P, P, P, P, P, None) == 0
        result += take()
for T, k, W in {ROWS + ROWS_LARGE!r}:
    for token in (0, 1):
        for slot in (0, 1):
            p = F.ExpertsParams(T, k, 8, W, W, W, W, W, token, slot, 0)
            assert lib.nvfp4_experts_sort(P, C.byref(p), P, P, P, P, 1 << 30, None) == 0
            assert lib.nvfp4_experts_spread(P, C.byref(p), P, P, None) == 0
            assert lib.nvfp4_experts_combine(P, C.byref(p), P, P, None, P, None) == 0
            assert lib.nvfp4_experts_combine_backward(P, C.byref(p), P, P, P, P, P, None) == 0
            result += take()
""")
    out = subprocess.run(["nm", "-D", str(build.SO)], text=True, capture_output=True, check=True).stdout
    base = int(re.search(r"(\w+) T nvfp4_distill_step$", out, flags=re.M).group(1), 16)
    known = _kernels()
    reached = {known[base + at] for at in launched}
    assert len(known) == 52 + 42
    assert reached == set(known.values()), "\n".join(sorted(set(known.values()) - reached))

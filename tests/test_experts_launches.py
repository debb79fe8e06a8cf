"""CPU: no product that the header allows needs more workgroups than a launch has, by the calls' own launches."""
from . import _hip_calls


def test_many_experts_of_many_columns_are_launched():
    """Tiles for every expert and every group of columns, were they all used, would be more threads than the 2^32 - 1 of a launch."""
    made = _hip_calls.run("""
from paper_2512_02010_amd import finetune as F
lib, result = F.lib(), []
for slots, N, E, K in ((5000, 1 << 22, 1024, 32), (4200, 1 << 22, 1024, 1024), (3000, 1 << 22, 1000, 32), (20000, (1 << 22) - 7, 1024, 256),
                       (1 << 30, 1 << 22, 1024, 1 << 22), (1 << 30, 1 << 22, 1, 32)):
    for dtype in (0, 1):
        for out in (0, 1):
            p = F.ProductParams(1000, K, N, E, slots, K, N, dtype, out, 0)
            p.ld_out = min(N, (1 << 40) // slots)
            p.out = min(N, p.ld_out)
            rc = lib.nvfp4_experts_product(P, C.byref(p), P, P, P, P, P, P, None)
            result.append(((slots, N, E, K, dtype, out), rc, [(c[0], c[3]) for c in calls() if c[0] == "launch"]))
""")
    for what, rc, launches in made:
        assert rc == 0 and len(launches) == 1, (what, rc)
        assert 0 < launches[0][1] <= (2 ** 32 - 1) // 64, (what, launches)

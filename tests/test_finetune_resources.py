"""CPU: no kernel of the adapters keeps anything in scratch memory, by the compiler's report."""
from .test_finetune_host import _report


def test_no_kernel_of_the_adapters_spills():
    kernels = {k: v for k, v in _report("adapters.hip").items() if "LDS" in v}
    assert sum("k_expand" in k for k in kernels) == 36
    spilled = {k: v["ScratchSize"] for k, v in kernels.items() if v["ScratchSize"]}
    assert not spilled, spilled

"""CPU: refusals of adapters and distillation that name what is wrong."""
import ctypes as C

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2512_02010_amd import finetune as F

from .test_finetune_abi import _adapters, _backward, _distill, _distill_calls, _forward


@pytest.mark.parametrize("temperature", [2.0 ** -127, 4.2e-39, 2.9e-39, 1e-39, 2.0 ** -149])
def test_temperatures_that_are_no_normal_numbers(temperature):
    """Below 4.24e-39 log2(e) / temperature is infinite in fp32 and every result was NaN; fp32's least normal number, 2^-126, is
    the least temperature."""
    assert C.c_float(temperature).value > 0
    for call, _ in _distill_calls():
        assert call(_distill(temperature=temperature)) == 4
        assert call(_distill(rows=0, temperature=2.0 ** -126)) == 0


def test_sizes_are_named_before_missing_pointers():
    """A tensor without elements has no address, nor has the workspace of a call whose sizes are refused: the status is the sizes'."""
    for call, more in ((_forward, {}), (_backward, dict(ld_base=64, ld_out=64))):
        for bad in (dict(inp=60, ld_x=60), dict(rank=0), dict(rank=129), dict(adapters=0), dict(adapters=2049), dict(out=0), dict(tokens=1 << 24)):
            assert call(_adapters(**{**more, **bad}), a=None, b=None, scales=None, workspace=None, room=0) == 2, bad
        assert call(_adapters(**more), workspace=None) == 1 and call(_adapters(**more), a=None) == 1
    for call, names in _distill_calls():
        for bad in (dict(vocab=0, ld=0), dict(top=0), dict(top=1025), dict(rows=-1)):
            assert call(_distill(**bad), **dict.fromkeys(names)) == 2, bad
        assert call(_distill(), **dict.fromkeys(names)) == 1


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_a_workspace_of_another_device():
    """Refused as every other operand of another device is.  (Tensors without memory stand for those of two devices.)"""
    with FakeTensorMode():
        def zeros(*shape, dtype=torch.bfloat16, device="cuda:0"):
            return torch.empty(shape, dtype=dtype, device=device)

        x, base, a, b = zeros(4, 64), zeros(4, 32), zeros(2, 8, 64), zeros(2, 32, 8)
        which, scales, h = zeros(4, dtype=torch.int32), zeros(2, dtype=torch.float32), zeros(4, 8, dtype=torch.float32)
        workspace = zeros(1 << 20, dtype=torch.uint8, device="cuda:1")
    with pytest.raises(AssertionError, match="workspace must be on the device of the others"):
        F.nvfp4_adapters_forward(x, base, a, b, which, scales, workspace=workspace)
    with pytest.raises(AssertionError, match="workspace must be on the device of the others"):
        F.nvfp4_adapters_backward(base, x, h, a, b, which, scales, workspace=workspace)

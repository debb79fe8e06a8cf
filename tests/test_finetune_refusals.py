"""CPU: refusals of adapters and distillation that name what is wrong."""
import ctypes as C

import pytest

from paper_2512_02010_amd import finetune as F

from .test_finetune_abi import P, _distill, _distill_calls


@pytest.mark.parametrize("temperature", [2.0 ** -127, 4.2e-39, 2.9e-39, 1e-39, 2.0 ** -149])
def test_temperatures_that_are_no_normal_numbers(temperature):
    """Below 4.24e-39 log2(e) / temperature is infinite in fp32 and every result was NaN; fp32's least normal number, 2^-126, is
    the least temperature."""
    assert C.c_float(temperature).value > 0
    for call, _ in _distill_calls():
        assert call(_distill(temperature=temperature)) == 4
        assert call(_distill(rows=0, temperature=2.0 ** -126)) == 0

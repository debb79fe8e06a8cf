"""Recovering, and serving, a model whose weights are quantized to NVFP4.

Low-rank adapters of many requests at once beside a shared projection, and distillation from a teacher's top logits: the
entry points of ``include/finetune/nvfp4_finetune.h`` under their C names, with output allocation, checks of arguments and errors
as in :mod:`.binding` (``Nvfp4Error`` for a status, ``AssertionError`` for tensors that do not fit together).
``adapted_fprop`` and ``adapted_backward`` string them together with the quantized layer of :mod:`.linear`.

Tensors live on the current device; matrices may have a stride from row to row.  With ``stream=None`` the work goes to the
current stream.  A workspace is allocated per call unless one is lent (``adapters_workspace``).
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as B
from . import linear as L

INDEX_I32, INDEX_I64 = 0, 1
ENTRY_POINTS = ("nvfp4_adapters_workspace_bytes", "nvfp4_adapters_forward", "nvfp4_adapters_backward", "nvfp4_distill_forward",
                "nvfp4_distill_backward", "nvfp4_distill_step", "nvfp4_weight_product", "nvfp4_experts_product",
                "nvfp4_experts_workspace_bytes", "nvfp4_experts_sort", "nvfp4_experts_spread", "nvfp4_experts_combine",
                "nvfp4_experts_combine_backward")        # (the last seven: experts.py)


class AdaptersParams(C.Structure):
    """Mirror of ``nvfp4_adapters_params``."""
    _fields_ = [("tokens", C.c_int64), ("inp", C.c_int64), ("out", C.c_int64), ("adapters", C.c_int64), ("rank", C.c_int64),
                ("ld_x", C.c_int64), ("ld_base", C.c_int64), ("ld_out", C.c_int64), ("ld_dy", C.c_int64), ("out_dtype", C.c_uint32)]


class DistillParams(C.Structure):
    """Mirror of ``nvfp4_distill_params``."""
    _fields_ = [("rows", C.c_int64), ("vocab", C.c_int64), ("ld", C.c_int64), ("top", C.c_int64), ("temperature", C.c_float),
                ("x_dtype", C.c_uint32), ("teacher_dtype", C.c_uint32), ("index_dtype", C.c_uint32)]


class ProductParams(C.Structure):
    """Mirror of ``nvfp4_product_params``."""
    _fields_ = [("rows", C.c_int64), ("inp", C.c_int64), ("out", C.c_int64), ("experts", C.c_int64), ("slots", C.c_int64),
                ("ld_x", C.c_int64), ("ld_out", C.c_int64), ("x_dtype", C.c_uint32), ("out_dtype", C.c_uint32), ("flags", C.c_uint32)]


class ExpertsParams(C.Structure):
    """Mirror of ``nvfp4_experts_params``."""
    _fields_ = [("tokens", C.c_int64), ("top", C.c_int64), ("experts", C.c_int64), ("width", C.c_int64), ("ld_token", C.c_int64),
                ("ld_base", C.c_int64), ("ld_slot", C.c_int64), ("ld_dslot", C.c_int64), ("token_dtype", C.c_uint32),
                ("slot_dtype", C.c_uint32), ("index_dtype", C.c_uint32)]


_lib = None


def lib() -> C.CDLL:
    """The library with these entry points declared (raises if it has not been built)."""
    global _lib
    if _lib is None:
        library = B.lib()
        vp, size = C.c_void_p, C.c_size_t
        a, d, w, e = (C.POINTER(p) for p in (AdaptersParams, DistillParams, ProductParams, ExpertsParams))
        for name, result, arguments in (
                ("nvfp4_adapters_workspace_bytes", size, [a, C.c_int]),
                ("nvfp4_adapters_forward", C.c_int, [vp, a] + [vp] * 8 + [size, vp]),
                ("nvfp4_adapters_backward", C.c_int, [vp, a] + [vp] * 11 + [size, vp]),
                ("nvfp4_distill_forward", C.c_int, [vp, d] + [vp] * 5),
                ("nvfp4_distill_backward", C.c_int, [vp, d] + [vp] * 6),
                ("nvfp4_distill_step", C.c_int, [vp, d] + [vp] * 6),
                ("nvfp4_weight_product", C.c_int, [vp, w] + [vp] * 5),
                ("nvfp4_experts_product", C.c_int, [vp, w] + [vp] * 7),
                ("nvfp4_experts_workspace_bytes", size, [e]),
                ("nvfp4_experts_sort", C.c_int, [vp, e] + [vp] * 4 + [size, vp]),
                ("nvfp4_experts_spread", C.c_int, [vp, e] + [vp] * 3),
                ("nvfp4_experts_combine", C.c_int, [vp, e] + [vp] * 5),
                ("nvfp4_experts_combine_backward", C.c_int, [vp, e] + [vp] * 6)):
            function = getattr(library, name)
            function.restype, function.argtypes = result, arguments
        _lib = library
    return _lib


_native = None


def native():
    """The module of ``csrc/python.cpp``, connected to these entry points."""
    global _native
    if _native is None:
        module, library = B.native(), lib()
        module.connect_finetune(*(C.cast(getattr(library, name), C.c_void_p).value for name in ENTRY_POINTS))
        _native = module
    return _native


def _allocate():
    return None if B.OUTPUT_ALLOCATOR is B._device_empty else B.OUTPUT_ALLOCATOR


def _handle(stream):
    return None if stream is None else B._stream(stream)


# ---- adapters ---------------------------------------------------------------------------------

def adapters_workspace(tokens: int, inp: int, out: int, adapters: int, rank: int, backward: bool, device="cuda") -> torch.Tensor:
    """A workspace for nvfp4_adapters_forward or _backward with these sizes; one serves the calls issued on one stream."""
    p = AdaptersParams(tokens, inp, out, adapters, rank, inp, inp, inp, out, 0)
    need = lib().nvfp4_adapters_workspace_bytes(C.byref(p), int(backward))
    if need == 0:
        raise B.Nvfp4Error(2, "nvfp4_adapters_workspace_bytes")
    return torch.empty(need, dtype=torch.uint8, device=device)


def nvfp4_adapters_forward(x: torch.Tensor, base: torch.Tensor | None, a: torch.Tensor, b: torch.Tensor, which: torch.Tensor,
                           scales: torch.Tensor, want_h: bool = False, out: torch.Tensor | None = None,
                           workspace: torch.Tensor | None = None, stream=None):
    """base [T][N] (BF16 or fp32; None for 0) plus scales[l] B_l A_l x_t of every token's adapter l = which[t], -1 for none.

    x [T][K] BF16, a [L][r][K] and b [L][N][r] BF16, which [T] int32, scales [L] fp32.  ``out`` may be ``base``.  With ``want_h``
    also h [T][r] fp32, for the backward pass."""
    return (_native or native()).adapters_forward(x, base, a, b, which, scales, want_h, out, workspace, _allocate(),
                                                  _handle(stream))


def nvfp4_adapters_backward(dy: torch.Tensor, x: torch.Tensor, h: torch.Tensor, a: torch.Tensor, b: torch.Tensor,
                            which: torch.Tensor, scales: torch.Tensor, dx_base: torch.Tensor | None = None, want_dx: bool = True,
                            out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None):
    """(dx [T][K] BF16, da [L][r][K] fp32, db [L][N][r] fp32) from dy [T][N] BF16 and the forward pass' x and h.  dx_base is the
    gradient through the shared projection, and ``out`` (for dx) may be it; without ``want_dx`` dx is None."""
    return (_native or native()).adapters_backward(dy, x, h, a, b, which, scales, dx_base, want_dx, out, workspace, _allocate(),
                                                   _handle(stream))


# ---- distillation -----------------------------------------------------------------------------

def nvfp4_distill_forward(logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, temperature: float = 1.0, stream=None):
    """(loss [T], lse [T]), fp32: the divergence of logits [T][V] (BF16 or fp32) from the teacher's logits [T][k] (BF16 or
    fp32) at the words index [T][k] (int32 or int64; outside [0, V): no entry)."""
    return (_native or native()).distill_forward(logits, teacher, index, temperature, _allocate(), _handle(stream))


def nvfp4_distill_backward(logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, lse: torch.Tensor,
                           weight: torch.Tensor | None = None, temperature: float = 1.0, out: torch.Tensor | None = None,
                           stream=None) -> torch.Tensor:
    """The gradient for the logits, in their type and with their strides, of the losses' sum with weight [T] (None: 1).
    ``out`` may be ``logits``."""
    return (_native or native()).distill_backward(logits, teacher, index, temperature, lse, weight, out, _allocate(),
                                                  _handle(stream))


def nvfp4_distill_step(logits: torch.Tensor, teacher: torch.Tensor, index: torch.Tensor, weight: torch.Tensor | None = None,
                       temperature: float = 1.0, out: torch.Tensor | None = None, stream=None):
    """(loss [T] fp32, without the weight, and the gradient) in one call."""
    return (_native or native()).distill_step(logits, teacher, index, temperature, weight, out, _allocate(), _handle(stream))


# ---- a quantized layer with adapters ------------------------------------------------------------

def adapted_fprop(x: torch.Tensor, qw: dict, a: torch.Tensor, b: torch.Tensor, which: torch.Tensor, scales: torch.Tensor,
                  want_h: bool = False, workspace: torch.Tensor | None = None, weight_only: bool = False):
    """y [T][N] BF16 = x W^T of a quantized weight (``linear.quantize_weight``), with every token's adapter added; with
    ``want_h`` (y, h).  ``workspace`` and ``weight_only`` are those of ``linear.fprop``."""
    y = L.fprop(x, qw, workspace=workspace, weight_only=weight_only)
    return nvfp4_adapters_forward(x, y, a, b, which, scales, want_h=want_h, out=y)


def adapted_backward(dy: torch.Tensor, x: torch.Tensor, h: torch.Tensor, qw: dict, a: torch.Tensor, b: torch.Tensor,
                     which: torch.Tensor, scales: torch.Tensor, sr_seed: int, want_dx: bool = True,
                     workspace: torch.Tensor | None = None, weight_only: bool = False):
    """(dx, da, db) of ``adapted_fprop``; the weight itself stays as it is."""
    dx = L.dgrad(dy, qw, sr_seed, workspace=workspace, weight_only=weight_only) if want_dx else None
    return nvfp4_adapters_backward(dy, x, h, a, b, which, scales, dx_base=dx, want_dx=want_dx, out=dx)

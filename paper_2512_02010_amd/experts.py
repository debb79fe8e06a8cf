"""Serving and differentiating quantized weights with activations as they are: one projection, or those of many experts.

``nvfp4_weight_product`` multiplies BF16 or fp32 activations, unrounded, with an NVFP4 weight; ``nvfp4_experts_product`` does so with a
weight for each expert.  ``nvfp4_experts_sort``, ``_spread`` and ``_combine`` take tokens to their experts and back, with the gradients.  These are the
entry points of ``include/finetune/nvfp4_finetune.h`` under their C names, with output allocation, checks of arguments and
errors as in :mod:`.finetune`.  ``feed_forward`` and ``feed_forward_backward`` string them together to a layer of experts.

Tensors live on the current device; matrices may have a stride from row to row.  With ``stream=None`` the work goes to the
current stream.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as B
from . import finetune as F

_native = None


def native():
    """The module of ``csrc/python.cpp``, connected to these entry points."""
    global _native
    if _native is None:
        _native = F.native()
    return _native


# ---- products with activations as they are ------------------------------------------------------

def nvfp4_weight_product(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, alpha: torch.Tensor, out_dtype: int = B.OUT_BF16,
                         flags: int = 0, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x [T][K] (BF16 or fp32, as it is) times W^T of a weight [N][K] in NVFP4: codes [N][K/2], scales [N][K/16] (or
    [N/16][K/16] with ``flags=GEMM_B_TILE_SCALES``), alpha [1].  The type of ``out``, where it is given, is the result's."""
    return (_native or native()).weight_product(x, codes, scales, alpha, out_dtype, flags, out, F._allocate(), F._handle(stream))


def nvfp4_experts_product(x: torch.Tensor, begin: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, alpha: torch.Tensor,
                          token: torch.Tensor | None = None, out_dtype: int = B.OUT_BF16, flags: int = 0,
                          out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """[S][N]: row s, begin[e] <= s < begin[e + 1], is x[token[s]] (x[s] without ``token``) times the weight of expert e; codes
    [E][N][K/2], scales [E][N][K/16], alpha [E].  Rows in front of begin[0] and from begin[E] on are 0."""
    return (_native or native()).experts_product(x, token, begin, codes, scales, alpha, out_dtype, flags, out, F._allocate(),
                                                 F._handle(stream))


# ---- tokens to their experts, and back ----------------------------------------------------------

def experts_workspace(tokens: int, top: int, experts: int, device="cuda") -> torch.Tensor:
    """A workspace for nvfp4_experts_sort with these sizes; one serves the calls issued on one stream."""
    p = F.ExpertsParams(tokens, top, experts, 8, 8, 8, 8, 8, 0, 0, 0)
    need = F.lib().nvfp4_experts_workspace_bytes(C.byref(p))
    if need == 0:
        raise B.Nvfp4Error(2, "nvfp4_experts_workspace_bytes")
    return torch.empty(need, dtype=torch.uint8, device=device)


def nvfp4_experts_sort(ids: torch.Tensor, experts: int, workspace: torch.Tensor | None = None, stream=None):
    """(place [T][k], token [T * k], begin [experts + 1]), int32, of the experts ids [T][k] (int32 or int64; outside [0, experts): none)."""
    return (_native or native()).experts_sort(ids, experts, workspace, F._allocate(), F._handle(stream))


def nvfp4_experts_spread(x: torch.Tensor, place: torch.Tensor, out_dtype: int | None = None, out: torch.Tensor | None = None,
                         stream=None) -> torch.Tensor:
    """xs [T * k][W] of x [T][W]: every token's row at the places of its experts, 0 where a pair has none.  Its gradient is
    ``nvfp4_experts_combine`` without weights."""
    return (_native or native()).experts_spread(x, place, out_dtype, out, F._allocate(), F._handle(stream))


def nvfp4_experts_combine(ys: torch.Tensor, place: torch.Tensor, weights: torch.Tensor | None = None,
                          base: torch.Tensor | None = None, out_dtype: int | None = None, out: torch.Tensor | None = None,
                          stream=None) -> torch.Tensor:
    """base [T][W] (None for 0) plus the sum over j of weights[t][j] (None for 1) ys[place[t][j]].  The result has the type of
    ``base`` or ``out`` where there is one, else ``out_dtype`` or ys' own.  ``out`` may be ``base``."""
    return (_native or native()).experts_combine(ys, place, weights, base, out_dtype, out, F._allocate(), F._handle(stream))


def nvfp4_experts_combine_backward(dy: torch.Tensor, ys: torch.Tensor, place: torch.Tensor, weights: torch.Tensor,
                                   out: torch.Tensor | None = None, stream=None):
    """(dys [T * k][W] of ys' type, dweights [T][k] fp32) from dy [T][W].  ``out`` (for dys) may be ys."""
    return (_native or native()).experts_combine_backward(dy, ys, place, weights, out, F._allocate(), F._handle(stream))


# ---- a layer of experts -------------------------------------------------------------------------

def quantize_experts(w: torch.Tensor, select: int = B.SEL_46_MSE, block2d: bool = True) -> dict:
    """W [E][N][K] -> both packings and the tensor scale of every expert's weight, as ``linear.quantize_weight`` has one's."""
    E, N, K = w.shape
    lines = (lambda n: n // 16) if block2d else (lambda n: n)

    def u8(*shape):
        return torch.empty((E, *shape), dtype=torch.uint8, device=w.device)

    q = dict(codes_row=u8(N, K // 2), scales_row=u8(lines(N), K // 16), codes_col=u8(K, N // 2), scales_col=u8(lines(K), N // 16),
             alpha=torch.empty(E, dtype=torch.float32, device=w.device))
    workspace = B.new_workspace(w.device)
    for e in range(E):
        one = B.nvfp4_46_scale_quantize(w[e].contiguous(), workspace, layout=B.BOTH, select=select, want_choice=False, block2d=int(block2d))
        for name, all_ in q.items():
            all_[e].copy_(one[name].view(all_[e].shape))
    q.update(block2d=bool(block2d), shape=(E, N, K))
    return q


def experts_fprop(x, begin, q: dict, token=None, out_dtype: int = B.OUT_BF16) -> torch.Tensor:
    """Every row times its expert's W^T."""
    return nvfp4_experts_product(x, begin, q["codes_row"], q["scales_row"], q["alpha"], token, out_dtype,
                                 B.GEMM_B_TILE_SCALES if q["block2d"] else 0)


def experts_dgrad(dy, begin, q: dict, out_dtype: int = B.OUT_BF16) -> torch.Tensor:
    """... times its expert's W, for the gradient."""
    return nvfp4_experts_product(dy, begin, q["codes_col"], q["scales_col"], q["alpha"], None, out_dtype,
                                 B.GEMM_B_TILE_SCALES if q["block2d"] else 0)


def feed_forward(x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, up: dict, down: dict, base: torch.Tensor | None = None):
    """y_t = base_t + sum_j weights[t][j] W_down relu(W_up x_t) of the experts ids[t][j], and what the backward pass needs.  The rows in between have
    x's type."""
    dtype = B.x_dtype_of(x)
    place, token, begin = nvfp4_experts_sort(ids, up["shape"][0])
    h = experts_fprop(x, begin, up, token, dtype)
    ys = experts_fprop(torch.relu(h), begin, down, None, dtype)
    return nvfp4_experts_combine(ys, place, weights, base, out_dtype=dtype), (place, begin, h, ys)


def feed_forward_backward(dy: torch.Tensor, kept, weights: torch.Tensor, up: dict, down: dict):
    """(dx, dweights) of ``feed_forward``; the experts' weights stay as they are, and base's gradient is dy.  dx has dy's type, the rows in between that
    of x."""
    place, begin, h, ys = kept
    dtype = B.x_dtype_of(h)
    dys, dweights = nvfp4_experts_combine_backward(dy, ys, place, weights)
    # (not times the mask: a gradient that overflowed, times 0, would be NaN)
    dh = experts_dgrad(dys, begin, down, dtype).masked_fill_(h <= 0, 0)
    return nvfp4_experts_combine(experts_dgrad(dh, begin, up, dtype), place, out_dtype=B.x_dtype_of(dy)), dweights

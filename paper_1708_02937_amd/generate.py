"""Generating tokens with a layer of experts, on torch tensors: the calls of include/sdnn.h with their shapes read from the
tensors and their outputs allocated.

A 4-bit matrix is a ``torch.float4_e2m1fn_x2`` tensor of ``sdnn_groups_pitch(k)`` columns, two codes each, and a
``torch.float8_e8m0fnu`` tensor of ``sdnn_groups_scale_pitch(k)`` scales, one for each group of 32 columns.  Streams,
devices, memory, graphs and gradients are as in experts.py: work goes to the current stream of the tensors' device, every
function may be called while a graph is captured, and a tensor that requires a gradient is a ValueError.
"""

from __future__ import annotations

import torch

from . import _tensors
from .experts import _checked, _current, _elsewhere, _kind, _stream


def quantize_groups(x):
    """(codes, scales) of a float32 or bfloat16 tensor (..., rows, k) rounded to 4 bits with a scale for each group of 32
    columns; a matrix may have any row stride, a stack of them has to be contiguous."""
    device = x.get_device()
    if device < 0 or device != _current():
        return _elsewhere(quantize_groups, device, x)
    return _checked(_tensors.quantize_groups(x, _stream(device)))


def widen_groups(codes, scales, k: int, dtype=torch.bfloat16):
    """The (..., rows, k) values that a 4-bit matrix stands for, exactly, in float32 or bfloat16."""
    device = codes.get_device()
    if device < 0 or device != _current():
        return _elsewhere(widen_groups, device, codes, scales, k, dtype)
    return _checked(_tensors.widen_groups(codes, scales, k, _kind(dtype), _stream(device)))


def product_groups(x, w, w_scale, bias=None, ymax=None, dtype=None, out=None):
    """h(X W^T + bias) of a few dense rows X (m x k, float32 or bfloat16) and 4-bit W (n x k); h clamps to [0, ymax], None
    leaves values as they are.  dtype: the result's, x's if absent.  Every product is exact and sums are float32."""
    device = x.get_device()
    if device < 0 or device != _current():
        return _elsewhere(product_groups, device, x, w, w_scale, bias, ymax, dtype, out)
    return _checked(_tensors.product_groups(x, w, w_scale, bias, ymax, None if dtype is None else _kind(dtype), out,
                                            _stream(device)))

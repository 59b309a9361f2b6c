"""Generating tokens with a layer of experts, on torch tensors: the calls of include/sdnn.h with their shapes read from the
tensors and their outputs allocated.

A 4-bit matrix is a ``torch.float4_e2m1fn_x2`` tensor of ``sdnn_groups_pitch(k)`` columns, two codes each, and a
``torch.float8_e8m0fnu`` tensor of ``sdnn_groups_scale_pitch(k)`` scales, one for each group of 32 columns.  Streams,
devices, memory, graphs and gradients are as in experts.py: work goes to the current stream of the tensors' device, every
function may be called while a graph is captured, and a tensor that requires a gradient is a ValueError.
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from . import _tensors
from .experts import _SCORES, _checked, _current, _elsewhere, _kind, _stream


class Layer(NamedTuple):
    """A layer's result (tokens x width), and the experts that each token took (ids and weight as in Routes)."""

    out: torch.Tensor
    ids: torch.Tensor
    weight: torch.Tensor


class Tokens(NamedTuple):
    """The next tokens: ids (int32, -1 where a row has none), prob (their share of what was kept) and kept (int32: how many
    tokens were)."""

    ids: torch.Tensor
    prob: torch.Tensor
    kept: torch.Tensor


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


def experts_layer(x, gamma, router, k: int, w_in, w_in_scale, w_out, w_out_scale, inner: int, eps: float = 1e-6,
                  residual=None, live=None, score: str = "softmax", bias=None, groups: int = 1, groups_kept: int = 1,
                  group_best: int = 1, normalize: bool = True, factor: float = 1.0, out=None, ws=None) -> Layer:
    """A whole layer of experts for up to 16 tokens (x: tokens x width): s = x + residual, its RMS norm times gamma, the
    router's logits (router: experts x width, float32 or bfloat16) and choice (k, score, bias, groups, ... as in route),
    and s + the weighted sum of the chosen experts on the norm in 8 bits (weights as in experts_forward).

    Of layers of a few hundred columns, norm_quantize, route and experts_forward are faster from about 4 tokens on.

    live: a bool for each token; one that is False takes part in no expert, and its result is s.  out may be x or residual
    itself.  ws: a uint8 tensor of at least sdnn_experts_layer_workspace_size bytes (allocated if absent)."""
    device = x.get_device()
    if device < 0 or device != _current():
        return _elsewhere(experts_layer, device, x, gamma, router, k, w_in, w_in_scale, w_out, w_out_scale, inner, eps,
                          residual, live, score, bias, groups, groups_kept, group_best, normalize, factor, out, ws)
    if score not in _SCORES:
        raise ValueError("score must be 'softmax' or 'sigmoid'")
    return Layer._make(_checked(_tensors.experts_layer(x, gamma, router, k, w_in, w_in_scale, w_out, w_out_scale, inner,
                                                       eps, residual, live, _SCORES[score], bias, groups, groups_kept,
                                                       group_best, normalize, factor, out, ws, _stream(device))))


def sample(logits, uniform, temperature=None, top_k=None, top_p=None, min_p=None, ws=None) -> Tokens:
    """The next token of each row of logits (rows x vocabulary, float32 or bfloat16) for a uniform number each (float64,
    in [0, 1)): of the top_k largest (int32; 0: all), of the shortest run of those whose mass is top_p of theirs, and of those
    with at least min_p of the largest one's probability, all at that temperature (0: the largest logit); see sdnn_sample.

    temperature, top_p and min_p are float32 tensors with a value for each row; what is None is off (temperature: 1).
    ws: a uint8 tensor of at least sdnn_sample_workspace_size bytes (allocated if absent)."""
    device = logits.get_device()
    if device < 0 or device != _current():
        return _elsewhere(sample, device, logits, uniform, temperature, top_k, top_p, min_p, ws)
    return Tokens._make(_checked(_tensors.sample(logits, uniform, temperature, top_k, top_p, min_p, ws, _stream(device))))

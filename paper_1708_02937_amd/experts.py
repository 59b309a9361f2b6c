"""A layer of experts on 8-bit operands, on torch tensors: the calls of include/sdnn.h with their shapes read from the
tensors and their outputs allocated.

Codes are ``torch.float8_e4m3fn`` tensors of ``sdnn_blocks_pitch(k)`` columns and scales ``torch.float8_e8m0fnu``
tensors of ``sdnn_blocks_scale_pitch(k)`` columns.  Work goes to the current stream of the tensors' device; outputs and
workspaces come from torch's allocator on that stream.  Every function may be called while a graph is captured.
"""

from __future__ import annotations

import functools
from typing import NamedTuple

import torch

import paper_1708_02937_amd as sd

CODES = torch.float8_e4m3fn
SCALES = torch.float8_e8m0fnu
_TYPES = {torch.float32: 0, torch.bfloat16: 1}  # SDNN_TYPE_*
_SCORES = {"softmax": 0, "sigmoid": 1}  # SDNN_SCORE_*


class Routes(NamedTuple):
    """Where each token goes: ids and weight (tokens x chosen; id -1 and weight 0 where there is no expert), and the
    slots t * chosen + j sorted by expert (offsets: experts + 1 counts; order: the slots, then -1)."""

    ids: torch.Tensor
    weight: torch.Tensor
    offsets: torch.Tensor
    order: torch.Tensor


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _dense(t, name, dtype=None, device=None, shape=None):
    """Checks a matrix whose rows are contiguous; returns its row stride."""
    _need(t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] <= 1), f"{name} must be a matrix with contiguous rows")
    _need(t.is_cuda, f"{name} must be on the GPU")
    _need(t.dtype == dtype if dtype is not None else t.dtype in _TYPES, f"{name}: unsupported type {t.dtype}")
    _need(device is None or t.device == device, f"{name} is on another device")
    _need(shape is None or tuple(t.shape) == shape, f"{name} must have shape {shape}, not {tuple(t.shape)}")
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


def _packed(t, name, dtype, device, shape):
    _need(t.is_cuda and t.device == device, f"{name} must be on the other tensors' device")
    _need(t.dtype == dtype, f"{name} must be {dtype}, not {t.dtype}")
    _need(t.is_contiguous() and tuple(t.shape) == shape, f"{name} must be contiguous with shape {shape}, not "
          f"{tuple(t.shape)}")


def _pitches(k):
    blocks = -(-k // 128)
    return blocks * 128, -(-blocks // 4) * 4


def _on_device(f):
    """Runs f with the device of its first tensor current."""

    @functools.wraps(f)
    def call(x, *args, **kw):
        if not x.is_cuda:
            raise ValueError(f"{f.__name__} needs tensors on the GPU")
        if x.device.index == torch.cuda.current_device():
            return f(x, *args, **kw)
        with torch.cuda.device(x.device):
            return f(x, *args, **kw)

    return call


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


@_on_device
def quantize_blocks(x, block_rows: int = 1):
    """(codes, scales) of a float32 or bfloat16 tensor (..., rows, k), contiguous, in blocks of block_rows x 128:
    1 for activations, 128 for weights."""
    _need(x.dim() >= 2 and x.is_contiguous(), "x must be contiguous, (..., rows, k)")
    _need(x.dtype in _TYPES, f"x: unsupported type {x.dtype}")
    rows, k = x.shape[-2:]
    pitch, spitch = _pitches(k)
    count = x.numel() // (rows * k) if rows * k else 0
    scale_rows = rows if block_rows == 1 else -(-rows // 128)
    codes = torch.empty((*x.shape[:-1], pitch), dtype=CODES, device=x.device)
    scales = torch.empty((*x.shape[:-2], scale_rows, spitch), dtype=SCALES, device=x.device)
    sd.sdnn_quantize_blocks(count, rows, k, block_rows, _TYPES[x.dtype], x, k, codes, scales, _stream(x.device))
    return codes, scales


@_on_device
def norm_quantize(x, gamma, eps: float = 1e-6, residual=None, normed: bool = False, out_sum=None):
    """(codes, scales, sum, normed): RMS norm of x + residual, times gamma (float32), as a blocked 8-bit matrix.

    sum is x + residual in x's type (None without a residual; written to out_sum if given, which may be x or residual
    itself); normed is the normalised row in x's type (None unless asked for)."""
    device, (rows, k) = x.device, x.shape
    ldx = _dense(x, "x")
    _packed(gamma, "gamma", torch.float32, device, (k,))
    pitch, spitch = _pitches(k)
    codes = torch.empty((rows, pitch), dtype=CODES, device=device)
    scales = torch.empty((rows, spitch), dtype=SCALES, device=device)
    ldr = lds = 0
    if residual is not None:
        ldr = _dense(residual, "residual", x.dtype, device, (rows, k))
        if out_sum is None:
            out_sum = torch.empty((rows, k), dtype=x.dtype, device=device)
        lds = _dense(out_sum, "out_sum", x.dtype, device, (rows, k))
    z = torch.empty((rows, k), dtype=x.dtype, device=device) if normed else None
    sd.sdnn_norm_quantize(rows, k, _TYPES[x.dtype], x, ldx, residual, ldr, gamma, eps, out_sum, lds, z, k, codes,
                          scales, _stream(device))
    return codes, scales, out_sum, z


@_on_device
def product_blocks(a, a_scale, w, w_scale, k: int, bias=None, ymax=None, dtype=torch.bfloat16, out=None):
    """h(A W^T + bias) of blocked 8-bit A (m x k) and W (n x k); h clamps to [0, ymax], None leaves values as they
    are.  dtype float32 keeps every product exact; bfloat16 takes the 8-bit matrix instructions."""
    device, m, n = a.device, a.shape[0], w.shape[0]
    pitch, spitch = _pitches(k)
    _packed(a, "a", CODES, device, (m, pitch))
    _packed(a_scale, "a_scale", SCALES, device, (m, spitch))
    _packed(w, "w", CODES, device, (n, pitch))
    _packed(w_scale, "w_scale", SCALES, device, (-(-n // 128), spitch))
    if bias is not None:
        _packed(bias, "bias", torch.float32, device, (n,))
    _need(dtype in _TYPES, f"unsupported output type {dtype}")
    if out is None:
        out = torch.empty((m, n), dtype=dtype, device=device)
    ldy = _dense(out, "out", dtype, device, (m, n))
    sd.sdnn_product_blocks(m, n, k, a, a_scale, w, w_scale, bias, ymax is not None, 0.0 if ymax is None else ymax,
                           _TYPES[dtype], out, ldy, _stream(device))
    return out


@_on_device
def route(logits, k: int, score: str = "softmax", bias=None, groups: int = 1, groups_kept: int = 1,
          group_best: int = 1, normalize: bool = True, factor: float = 1.0) -> Routes:
    """The k best experts of each token (logits: tokens x experts, float32 or bfloat16); see sdnn_route."""
    device, (tokens, experts) = logits.device, logits.shape
    ldl = _dense(logits, "logits")
    _need(score in _SCORES, "score must be 'softmax' or 'sigmoid'")
    if bias is not None:
        _packed(bias, "bias", torch.float32, device, (experts,))
    ids = torch.empty((tokens, k), dtype=torch.int32, device=device)
    weight = torch.empty((tokens, k), dtype=torch.float32, device=device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
    order = torch.empty(tokens * k, dtype=torch.int32, device=device)
    need = sd.sdnn_route_workspace_size(tokens, experts, k)
    ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    sd.sdnn_route(tokens, experts, k, _SCORES[score], _TYPES[logits.dtype], logits, ldl, bias, groups, groups_kept,
                  group_best, bool(normalize), factor, ids, weight, offsets, order, ws, need, _stream(device))
    return Routes(ids, weight, offsets, order)


@_on_device
def experts_forward(a, a_scale, routes: Routes, w_in, w_in_scale, w_out, w_out_scale, width: int, inner: int,
                    residual=None, dtype=torch.bfloat16, out=None, ws=None):
    """residual + the weighted sum of each token's experts (gated by SiLU) on its blocked 8-bit row of A.

    w_in: codes (experts, 2, inner, pitch of width), gate then up; w_out: codes (experts, width, pitch of inner); both
    with 128-row blocks, as quantize_blocks(w, 128) gives them.  ws: a uint8 tensor of at least
    sdnn_experts_workspace_size bytes (allocated if absent)."""
    device, tokens, experts = a.device, a.shape[0], w_in.shape[0]
    ids, weight, offsets, order = routes
    _need(ids.dim() == 2, "ids must be tokens x chosen")
    chosen = ids.shape[1]
    pitch, spitch = _pitches(width)
    pitch_f, spitch_f = _pitches(inner)
    _packed(a, "a", CODES, device, (tokens, pitch))
    _packed(a_scale, "a_scale", SCALES, device, (tokens, spitch))
    _packed(ids, "ids", torch.int32, device, (tokens, chosen))
    _packed(weight, "weight", torch.float32, device, (tokens, chosen))
    _packed(offsets, "offsets", torch.int32, device, (experts + 1,))
    _packed(order, "order", torch.int32, device, (tokens * chosen,))
    _packed(w_in, "w_in", CODES, device, (experts, 2, inner, pitch))
    _packed(w_in_scale, "w_in_scale", SCALES, device, (experts, 2, -(-inner // 128), spitch))
    _packed(w_out, "w_out", CODES, device, (experts, width, pitch_f))
    _packed(w_out_scale, "w_out_scale", SCALES, device, (experts, -(-width // 128), spitch_f))
    _need(dtype in _TYPES, f"unsupported output type {dtype}")
    ldr = 0
    if residual is not None:
        ldr = _dense(residual, "residual", dtype, device, (tokens, width))
    if out is None:
        out = torch.empty((tokens, width), dtype=dtype, device=device)
    ldo = _dense(out, "out", dtype, device, (tokens, width))
    if ws is None:
        need = sd.sdnn_experts_workspace_size(tokens, width, inner, experts, chosen, _TYPES[dtype])
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _need(ws.is_cuda and ws.device == device and ws.dtype == torch.uint8 and ws.is_contiguous(),
              "ws must be a contiguous uint8 tensor on the same device")
    sd.sdnn_experts_forward(tokens, width, inner, experts, chosen, a, a_scale, ids, weight, offsets, order, w_in,
                            w_in_scale, w_out, w_out_scale, _TYPES[dtype], residual, ldr, out, ldo, ws, ws.numel(),
                            _stream(device))
    return out

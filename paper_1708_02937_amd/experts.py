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
_SMALL_PLAN = 8192  # slots up to which sdnn_route needs no workspace


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


def _dense(t, name, dtype, device, shape):
    """Checks a matrix of that type and shape on that device, with contiguous rows; returns its row stride."""
    if t.dtype is not dtype or t.device != device or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} of shape {shape} on {device}, not {t.dtype} of shape "
                         f"{tuple(t.shape)} on {t.device}")
    rows, cols = t.stride()
    if cols != 1 and shape[1] > 1:
        raise ValueError(f"{name} must have contiguous rows")
    return rows if shape[0] > 1 else max(rows, shape[1])


def _packed(t, name, dtype, device, shape):
    """Checks a contiguous tensor of that type and shape on that device; returns its address."""
    if t.dtype is not dtype or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, {dtype} of shape {shape} on {device}, not {t.dtype} of shape "
                         f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _type(dtype, name):
    if dtype not in _TYPES:
        raise ValueError(f"{name}: float32 or bfloat16, not {dtype}")
    return _TYPES[dtype]


def _pitches(k):
    blocks = -(-k // 128)
    return blocks * 128, -(-blocks // 4) * 4


def _on_device(f):
    """Runs f with the device of its first tensor current."""

    @functools.wraps(f)
    def call(x, *args, **kw):
        index = x.get_device()  # -1 on the host
        if index < 0:
            raise ValueError(f"{f.__name__} needs tensors on the GPU")
        if index == torch.cuda.current_device():
            return f(x, *args, **kw)
        with torch.cuda.device(index):
            return f(x, *args, **kw)

    return call


def _like(x, ld, shape):
    """An empty contiguous matrix of x's type and shape."""
    return torch.empty_like(x) if ld == shape[1] else torch.empty(shape, dtype=x.dtype, device=x.device)


def _stream(device):
    return torch._C._cuda_getCurrentRawStream(device.index)


def _call(status):
    if status:
        sd._check(status)


@_on_device
def quantize_blocks(x, block_rows: int = 1):
    """(codes, scales) of a float32 or bfloat16 tensor (..., rows, k), contiguous, in blocks of block_rows x 128:
    1 for activations, 128 for weights."""
    _need(x.dim() >= 2 and x.is_contiguous(), "x must be contiguous, (..., rows, k)")
    kind = _type(x.dtype, "x")
    rows, k = x.shape[-2:]
    pitch, spitch = _pitches(k)
    count = x.numel() // (rows * k) if rows * k else 0
    scale_rows = rows if block_rows == 1 else -(-rows // 128)
    codes = torch.empty((*x.shape[:-1], pitch), dtype=CODES, device=x.device)
    scales = torch.empty((*x.shape[:-2], scale_rows, spitch), dtype=SCALES, device=x.device)
    sd.sdnn_quantize_blocks(count, rows, k, block_rows, kind, x, k, codes, scales, _stream(x.device))
    return codes, scales


@_on_device
def norm_quantize(x, gamma, eps: float = 1e-6, residual=None, normed: bool = False, out_sum=None):
    """(codes, scales, sum, normed): RMS norm of x + residual, times gamma (float32), as a blocked 8-bit matrix.

    sum is x + residual in x's type (None without a residual; written to out_sum if given, which may be x or residual
    itself); normed is the normalised row in x's type (None unless asked for)."""
    shape, dtype, device = x.shape, x.dtype, x.device
    _need(len(shape) == 2, "x must be a matrix")
    rows, k = shape
    kind = _type(dtype, "x")
    ldx = _dense(x, "x", dtype, device, shape)
    g = _packed(gamma, "gamma", torch.float32, device, (k,))
    pitch, spitch = _pitches(k)
    codes = torch.empty((rows, pitch), dtype=CODES, device=device)
    scales = torch.empty((rows, spitch), dtype=SCALES, device=device)
    r = s = z = None
    ldr = lds = 0
    if residual is not None:
        ldr, r = _dense(residual, "residual", dtype, device, shape), residual.data_ptr()
        if out_sum is None:
            out_sum, lds = _like(x, ldx, shape), k
        else:
            lds = _dense(out_sum, "out_sum", dtype, device, shape)
        s = out_sum.data_ptr()
    else:
        _need(out_sum is None, "out_sum without a residual")
    out_normed = None
    if normed:
        out_normed = _like(x, ldx, shape)
        z = out_normed.data_ptr()
    _call(sd.lib.sdnn_norm_quantize(rows, k, kind, x.data_ptr(), ldx, r, ldr, g, eps, s, lds, z, k, codes.data_ptr(),
                                    scales.data_ptr(), _stream(device)))
    return codes, scales, out_sum, out_normed


@_on_device
def product_blocks(a, a_scale, w, w_scale, k: int, bias=None, ymax=None, dtype=torch.bfloat16, out=None):
    """h(A W^T + bias) of blocked 8-bit A (m x k) and W (n x k); h clamps to [0, ymax], None leaves values as they
    are.  dtype float32 keeps every product exact; bfloat16 takes the 8-bit matrix instructions."""
    device, m, n = a.device, a.shape[0], w.shape[0]
    pitch, spitch = _pitches(k)
    kind = _type(dtype, "dtype")
    pa = _packed(a, "a", CODES, device, (m, pitch))
    psa = _packed(a_scale, "a_scale", SCALES, device, (m, spitch))
    pw = _packed(w, "w", CODES, device, (n, pitch))
    psw = _packed(w_scale, "w_scale", SCALES, device, (-(-n // 128), spitch))
    pb = None if bias is None else _packed(bias, "bias", torch.float32, device, (n,))
    if out is None:
        out, ldy = torch.empty((m, n), dtype=dtype, device=device), n
    else:
        ldy = _dense(out, "out", dtype, device, (m, n))
    _call(sd.lib.sdnn_product_blocks(m, n, k, pa, psa, pw, psw, pb, ymax is not None, 0.0 if ymax is None else ymax,
                                     kind, out.data_ptr(), ldy, _stream(device)))
    return out


@_on_device
def route(logits, k: int, score: str = "softmax", bias=None, groups: int = 1, groups_kept: int = 1,
          group_best: int = 1, normalize: bool = True, factor: float = 1.0) -> Routes:
    """The k best experts of each token (logits: tokens x experts, float32 or bfloat16); see sdnn_route."""
    device, shape = logits.device, logits.shape
    _need(len(shape) == 2, "logits must be tokens x experts")
    tokens, experts = shape
    kind = _type(logits.dtype, "logits")
    ldl = _dense(logits, "logits", logits.dtype, device, shape)
    _need(score in _SCORES, "score must be 'softmax' or 'sigmoid'")
    _need(k >= 1, "k must be at least 1")
    b = None if bias is None else _packed(bias, "bias", torch.float32, device, (experts,))
    ids = torch.empty((tokens, k), dtype=torch.int32, device=device)
    weight = torch.empty((tokens, k), dtype=torch.float32, device=device)
    offsets = torch.empty(experts + 1, dtype=torch.int32, device=device)
    order = torch.empty(tokens * k, dtype=torch.int32, device=device)
    ws, need = None, 0
    if tokens * k > _SMALL_PLAN:
        need = sd.sdnn_route_workspace_size(tokens, experts, k)
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    _call(sd.lib.sdnn_route(tokens, experts, k, _SCORES[score], kind, logits.data_ptr(), ldl, b, groups, groups_kept,
                            group_best, bool(normalize), factor, ids.data_ptr(), weight.data_ptr(),
                            offsets.data_ptr(), order.data_ptr(), None if ws is None else ws.data_ptr(), need,
                            _stream(device)))
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
    kind = _type(dtype, "dtype")
    pitch, spitch = _pitches(width)
    pitch_f, spitch_f = _pitches(inner)
    pa = _packed(a, "a", CODES, device, (tokens, pitch))
    psa = _packed(a_scale, "a_scale", SCALES, device, (tokens, spitch))
    pi = _packed(ids, "ids", torch.int32, device, (tokens, chosen))
    pw = _packed(weight, "weight", torch.float32, device, (tokens, chosen))
    pf = _packed(offsets, "offsets", torch.int32, device, (experts + 1,))
    po = _packed(order, "order", torch.int32, device, (tokens * chosen,))
    p1 = _packed(w_in, "w_in", CODES, device, (experts, 2, inner, pitch))
    ps1 = _packed(w_in_scale, "w_in_scale", SCALES, device, (experts, 2, -(-inner // 128), spitch))
    p2 = _packed(w_out, "w_out", CODES, device, (experts, width, pitch_f))
    ps2 = _packed(w_out_scale, "w_out_scale", SCALES, device, (experts, -(-width // 128), spitch_f))
    pr, ldr = None, 0
    if residual is not None:
        ldr, pr = _dense(residual, "residual", dtype, device, (tokens, width)), residual.data_ptr()
    if out is None:
        out, ldo = torch.empty((tokens, width), dtype=dtype, device=device), width
    else:
        ldo = _dense(out, "out", dtype, device, (tokens, width))
    if ws is None:
        need = sd.sdnn_experts_workspace_size(tokens, width, inner, experts, chosen, kind)
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        _need(ws.device == device and ws.dtype is torch.uint8 and ws.is_contiguous(),
              "ws must be a contiguous uint8 tensor on the same device")
    _call(sd.lib.sdnn_experts_forward(tokens, width, inner, experts, chosen, pa, psa, pi, pw, pf, po, p1, ps1, p2, ps2,
                                      kind, pr, ldr, out.data_ptr(), ldo, ws.data_ptr(), ws.numel(), _stream(device)))
    return out

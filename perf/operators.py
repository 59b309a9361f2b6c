"""Performance cases of the operators of a layer of experts on 8-bit operands.

``norm``     residual addition, RMS norm, and an output in 8 bits with a scale for each block of 128 columns
``route``    scores, groups, the k best experts of each token, their weights, and the slots sorted by expert
``product``  matrix product of two 8-bit matrices with a scale for each block of 128
``experts``  the gated feed-forward products of the chosen experts and their weighted sum

Each case is one call a program makes while it serves a prompt or a single token.  ``listed()`` holds the named cases,
``draw()`` gives further ones of the same ranges, ``prepare()`` makes the inputs on the GPU from a seed, ``run()`` is
one call (in plain torch, or the library's where ``own`` is set), ``exact()`` the same result in 64 bits.

8-bit format: codes are e4m3 (no infinities), one row padded with zeros to a multiple of 128 columns; a block's scale is
a power of two, held as its exponent (e8m0), the least one (2^-126 at least) that brings the block's largest finite
magnitude to 448 or less; a row of scales is padded to a multiple of 4 with the scale of an empty block.  Blocks are
1 x 128 for activations and 128 x 128 for weights.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 128
EPS = 1e-6


def listed():
    return [
        # One token's hidden state between two layers: latency.
        dict(name="norm-token", op="norm", T=1, H=4096, dtype="bf16", residual=True, normed=True),
        # Single precision, a width and a count that are multiples of nothing, no residual.
        dict(name="norm-odd", op="norm", T=777, H=1001, dtype="f32", residual=False, normed=False),
        # A long prompt's activations, every output wanted: memory bandwidth.
        dict(name="norm-prompt", op="norm", T=16384, H=4096, dtype="bf16", residual=True, normed=True),
        # One token through a softmax router.
        dict(name="route-token", op="route", T=1, E=64, k=4, score="softmax", bias=False, groups=1, kept=1, best=1,
             dtype="f32", masked=0.0),
        # An odd batch with padding tokens (rows that are masked whole) and a balance bias.
        dict(name="route-odd", op="route", T=1021, E=60, k=5, score="sigmoid", bias=True, groups=1, kept=1, best=1,
             dtype="f32", masked=0.1),
        # A long prompt over many experts in groups: the scores' arithmetic and the sort of the slots.
        dict(name="route-prompt", op="route", T=32768, E=256, k=8, score="sigmoid", bias=True, groups=8, kept=4,
             best=2, dtype="f32", masked=0.0),
        # One token through a layer with bias and ReLU: the weights' bytes.
        dict(name="product-token", op="product", M=1, N=4096, K=4096, dtype="f32", bias=True, relu=True),
        # The ragged batch of an MLP whose widths are multiples of nothing.
        dict(name="product-odd", op="product", M=777, N=2999, K=1001, dtype="f32", bias=True, relu=True),
        # A long batch through a wide layer: the matrix cores' rate.
        dict(name="product-prompt", op="product", M=8192, N=16384, K=4096, dtype="bf16", bias=False, relu=False),
        # One token through its 8 of 64 experts: the chosen weights' bytes.
        dict(name="experts-token", op="experts", T=1, H=4096, F=1024, E=64, k=8, dtype="bf16", residual=True,
             masked=0.0),
        # A small odd batch with padding tokens; widths that end inside a block; experts with few rows each.
        dict(name="experts-odd", op="experts", T=333, H=2001, F=701, E=24, k=3, dtype="bf16", residual=False,
             masked=0.1),
        # A long prompt, every expert busy: the matrix cores' rate over uneven groups.
        dict(name="experts-prompt", op="experts", T=8192, H=4096, F=1024, E=64, k=8, dtype="bf16", residual=True,
             masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of an operator, over its whole range of sizes, no dearer than the operator's largest listed one."""
    op = rng.choice(["norm", "route", "product", "experts"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        c = _draw(rng, op)
        if _cost(c) <= most:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 300)


def _draw(rng, op):
    dtype = rng.choice(["f32", "bf16"])
    if op == "norm":
        return dict(op=op, T=_log(rng, 1, 16384), H=_log(rng, 64, 16384), dtype=dtype, residual=rng.random() < 0.7,
                    normed=rng.random() < 0.5)
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * _log(rng, max(2, 4 // groups), 512 // groups)
        kept = rng.randint(1, groups)
        return dict(op=op, T=_log(rng, 1, 32768), E=E, k=rng.randint(1, min(8, E // groups * kept)),
                    score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups, kept=kept,
                    best=rng.randint(1, 2), dtype=dtype, masked=rng.choice([0.0, 0.1]))
    if op == "product":
        return dict(op=op, M=_log(rng, 1, 8192), N=_log(rng, 64, 16384), K=_log(rng, 64, 16384), dtype=dtype,
                    bias=rng.random() < 0.5, relu=rng.random() < 0.5)
    E = _log(rng, 4, 64)
    return dict(op=op, T=_log(rng, 1, 8192), H=_log(rng, 256, 4096), F=_log(rng, 128, 2048), E=E,
                k=rng.randint(1, min(8, E)), dtype="bf16", residual=rng.random() < 0.5, masked=rng.choice([0.0, 0.1]))


def work(case):
    op = case["op"]
    size = 4 if case["dtype"] == "f32" else 2
    if op == "norm":
        cells, tensors = case["T"] * case["H"], 1 + 2 * case["residual"] + case["normed"]
        return {"bytes": cells * (tensors * size + 1) + cells / BLOCK + 4 * case["H"], "flops": 8 * cells}
    if op == "route":
        cells, slots = case["T"] * case["E"], case["T"] * case["k"]
        return {"bytes": cells * size + 12 * slots + 4 * case["E"] * (2 if case["bias"] else 1), "flops": 8 * cells}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * K + M * N * size + (M * K + N * K / BLOCK) / BLOCK, "flops": 2 * M * N * K}
    T, H, F, E, k = (case[x] for x in ("T", "H", "F", "E", "k"))
    slots = T * k * (1 - case["masked"])
    busy = E * (1 - (1 - k / E) ** T)  # experts that an even router reaches
    return {"bytes": busy * 3 * F * H + T * H * (1 + size * (1 + case["residual"])) + 12 * T * k,
            "flops": 6 * slots * F * H}


# ------------------------------------------------------------------------------------------------ inputs


def _pad(n, to):
    return -(-n // to) * to


def _powers(codes):
    """The powers of two that e8m0 codes (1 to 254) stand for."""
    return (codes.view(torch.uint8).to(torch.int32) << 23).view(torch.float32)


def _quantize(z, rows):
    """(codes, scale) of a (..., R, K) float32 tensor in blocks of rows x 128."""
    R, K = z.shape[-2:]
    z = torch.nn.functional.pad(z, (0, _pad(K, BLOCK) - K, 0, _pad(R, rows) - R))
    tiles = z.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, rows))  # (..., R/rows, rows, K/128, 128)
    size = torch.where(tiles.isfinite(), tiles.abs(), 0.0).amax(dim=(-3, -1)).view(torch.int32)
    code = ((size >> 23) - 8 + ((size & 0x7FFFFF) > 0x600000)).clamp(min=1)
    inverse = ((254 - code) << 23).view(torch.float32)[..., :, None, :, None]
    q = tiles * inverse
    q = torch.where(q.isfinite(), q, float("nan")).flatten(-4, -3).flatten(-2)[..., :R, :].to(torch.float8_e4m3fn)
    scale = torch.nn.functional.pad(code.to(torch.uint8), (0, _pad(code.shape[-1], 4) - code.shape[-1]), value=1)
    return q.contiguous(), scale.contiguous().view(torch.float8_e8m0fnu)


def _values(q, scale, rows):
    """The float32 values that (..., R, pitch) codes in blocks of rows x 128 stand for."""
    s = _powers(scale)[..., :q.shape[-1] // BLOCK]
    if rows > 1:
        s = s.repeat_interleave(rows, dim=-2)[..., :q.shape[-2], :]
    return (q.to(torch.float32).unflatten(-1, (-1, BLOCK)) * s[..., None]).flatten(-2)


def _hidden(g, T, H):
    """Hidden states: normal, with a few columns ten times as wide, as trained models have them."""
    x = torch.randn((T, H), generator=g, device=DEV)
    return x * torch.where(torch.rand(H, generator=g, device=DEV) < 0.01, 10.0, 1.0)


def _weights(g, shape):
    return _quantize(torch.randn(shape, generator=g, device=DEV) / math.sqrt(shape[-1]), BLOCK)


def _logits(g, T, E, masked):
    """Router logits with experts of uneven popularity; masked tokens have no expert at all."""
    x = 1.5 * torch.randn((T, E), generator=g, device=DEV) + 0.5 * torch.randn(E, generator=g, device=DEV)
    return torch.where(torch.rand((T, 1), generator=g, device=DEV) < masked, -math.inf, x)


def _plan(ids, E):
    """(offsets, order): how many slots come before each expert's, and the slots sorted by expert (-1 at the end)."""
    flat = ids.reshape(-1).to(torch.int64)
    flat = torch.where(flat < 0, E, flat)
    count = torch.zeros(E + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, flat, torch.ones_like(flat))
    offsets = torch.nn.functional.pad(count[:E].cumsum(0), (1, 0))
    order = torch.sort(flat, stable=True)[1]
    order = torch.where(torch.arange(flat.numel(), device=ids.device) < offsets[E], order, -1)
    return offsets.to(torch.int32), order.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)
    s = dict(case)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "norm":
        T, H = case["T"], case["H"]
        s["x"] = _hidden(g, T, H).to(dtype)
        s["r"] = _hidden(g, T, H).to(dtype) if case["residual"] else None
        s["gamma"] = 1 + 0.1 * torch.randn(H, generator=g, device=DEV)
    elif case["op"] == "route":
        s["logits"] = _logits(g, case["T"], case["E"], case["masked"]).to(dtype)
        # a balance bias moves in steps of a thousandth
        steps = torch.randint(-100, 101, (case["E"],), generator=g, device=DEV)
        s["b"] = steps.to(torch.float32) * 1e-3 if case["bias"] else None
    elif case["op"] == "product":
        s["a"], s["sa"] = _quantize(_hidden(g, case["M"], case["K"]), 1)
        s["w"], s["sw"] = _weights(g, (case["N"], case["K"]))
        s["b"] = 0.1 * torch.randn(case["N"], generator=g, device=DEV) if case["bias"] else None
    else:
        T, H, F, E, k = (case[x] for x in ("T", "H", "F", "E", "k"))
        s["a"], s["sa"] = _quantize(_hidden(g, T, H), 1)
        s["w_in"], s["sw_in"] = _weights(g, (E, 2, F, H))
        s["w_out"], s["sw_out"] = _weights(g, (E, H, F))
        s["r"] = _hidden(g, T, H).to(dtype) if case["residual"] else None
        logits = _logits(g, T, E, case["masked"])
        top, ids = torch.topk(logits, k, dim=1)
        s["ids"] = torch.where(top > -math.inf, ids, -1).to(torch.int32)
        s["weight"] = torch.where(top > -math.inf, torch.softmax(top, dim=1), 0.0)
        s["offsets"], s["order"] = _plan(s["ids"], E)
    return s


# ------------------------------------------------------------------------------------------------ one call


def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _plain_norm(s):
    x = s["x"].to(torch.float32)
    if s["r"] is not None:
        x = x + s["r"].to(torch.float32)
    z = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * s["gamma"]
    q, scale = _quantize(z, 1)
    out = {"q": q, "scale": scale}
    if s["r"] is not None:
        out["sum"] = x.to(s["x"].dtype)
    if s["normed"]:
        out["normed"] = z.to(s["x"].dtype)
    return out


def _plain_route(s):
    # The scores are held in 64 bits: which experts are chosen is then the same whatever the order of a sum.
    l = s["logits"].to(torch.float64)
    T, E = l.shape
    there = l > -math.inf
    if s["score"] == "softmax":
        l = torch.where(there, l, -math.inf)
        p = torch.where(there, torch.exp(l - l.amax(dim=1, keepdim=True)), 0.0)
        score = p / p.sum(dim=1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-l))
    choice = score if s["b"] is None else score + s["b"].to(torch.float64)
    choice = torch.where(there, choice, -math.inf)
    if s["groups"] > 1:
        best = torch.sort(choice.view(T, s["groups"], -1), dim=2, descending=True)[0][:, :, :s["best"]]
        total = torch.where(best > -math.inf, best, 0.0).sum(dim=2)
        total = torch.where(best[:, :, 0] > -math.inf, total, -math.inf)
        kept = torch.sort(total, dim=1, descending=True, stable=True)[1][:, :s["kept"]]
        keep = torch.zeros_like(total, dtype=torch.bool).scatter_(1, kept, True)
        choice = torch.where(keep.repeat_interleave(E // s["groups"], dim=1), choice, -math.inf)
    top, ids = torch.sort(choice, dim=1, descending=True, stable=True)
    top, ids = top[:, :s["k"]], ids[:, :s["k"]]
    chosen = top > -math.inf
    weight = torch.where(chosen, score.gather(1, ids), 0.0)
    total = weight.sum(dim=1, keepdim=True)
    weight = torch.where(total > 0, weight / total, 0.0).to(torch.float32)
    ids = torch.where(chosen, ids, -1).to(torch.int32)
    offsets, order = _plan(ids, E)
    return {"ids": ids, "weight": weight, "offsets": offsets, "order": order}


def _plain_product(s):
    y = _values(s["a"], s["sa"], 1) @ _values(s["w"], s["sw"], BLOCK).t()
    if s["b"] is not None:
        y = y + s["b"]
    if s["relu"]:
        y = y.clamp(min=0)
    return y.to(DTYPES[s["dtype"]])


def _plain_experts(s):
    T, F, H, E, k = (s[x] for x in ("T", "F", "H", "E", "k"))
    x = _values(s["a"], s["sa"], 1)
    ids, w_in, sw_in, w_out, sw_out = s["ids"].reshape(-1).long(), s["w_in"], s["sw_in"], s["w_out"], s["sw_out"]
    slots = torch.arange(T * k, device=DEV)
    if T * k <= E:  # few slots: each takes its own expert's weights
        at, lanes = ids.clamp(min=0), slots[:, None]
        w_in, w_out = w_in.view(torch.uint8)[at].view(w_in.dtype), w_out.view(torch.uint8)[at].view(w_out.dtype)
        sw_in, sw_out = sw_in.view(torch.uint8)[at], sw_out.view(torch.uint8)[at]
        there = (ids >= 0)[:, None]
    else:  # the slots of an expert side by side, every expert padded to the fullest one
        offsets = s["offsets"].long()
        count = offsets[1:] - offsets[:-1]
        lane = torch.arange(max(1, int(count.max())), device=DEV)
        there = lane < count[:, None]
        lanes = s["order"].long()[torch.where(there, offsets[:-1, None] + lane, 0)]
        lanes = torch.where(there, lanes, 0)
    rows = torch.where(there[..., None], x[lanes // k], 0.0).transpose(1, 2).contiguous()
    z = torch.bmm(_values(w_in, sw_in, BLOCK).flatten(1, 2), rows)  # (experts, 2 F, lanes)
    gate, up = z[:, :F], z[:, F:]
    p = gate / (1 + torch.exp(-gate)) * up
    p = _values(*_quantize(p.transpose(1, 2), 1), 1).transpose(1, 2).contiguous()
    o = torch.bmm(_values(w_out, sw_out, BLOCK), p).transpose(1, 2)  # (experts, lanes, H)
    weight = torch.where(there, s["weight"].reshape(-1)[lanes], 0.0)
    part = torch.zeros((T * k + 1, H), device=DEV)
    part[torch.where(there, lanes, T * k)] = o * weight[..., None]
    out = part[:T * k].view(T, k, H).sum(dim=1)
    if s["r"] is not None:
        out = out + s["r"].to(torch.float32)
    return out.to(DTYPES[s["dtype"]])


_plain = {"norm": _plain_norm, "route": _plain_route, "product": _plain_product, "experts": _plain_experts}


def _own_norm(s):
    import paper_1708_02937_amd as sd

    q, scale, total, normed = sd.norm_quantize(s["x"], s["gamma"], EPS, residual=s["r"], normed=s["normed"])
    out = {"q": q, "scale": scale}
    if total is not None:
        out["sum"] = total
    if normed is not None:
        out["normed"] = normed
    return out


def _own_route(s):
    import paper_1708_02937_amd as sd

    r = sd.route(s["logits"], s["k"], score=s["score"], bias=s["b"], groups=s["groups"], groups_kept=s["kept"],
                 group_best=s["best"])
    return {"ids": r.ids, "weight": r.weight, "offsets": r.offsets, "order": r.order}


def _own_product(s):
    import paper_1708_02937_amd as sd

    return sd.product_blocks(s["a"], s["sa"], s["w"], s["sw"], s["K"], bias=s["b"],
                             ymax=math.inf if s["relu"] else None, dtype=DTYPES[s["dtype"]])


def _own_experts(s):
    import paper_1708_02937_amd as sd

    routes = sd.Routes(s["ids"], s["weight"], s["offsets"], s["order"])
    return sd.experts_forward(s["a"], s["sa"], routes, s["w_in"], s["sw_in"], s["w_out"], s["sw_out"], s["H"],
                              s["F"], residual=s["r"], dtype=DTYPES[s["dtype"]])


_own = {"norm": _own_norm, "route": _own_route, "product": _own_product, "experts": _own_experts}


# ------------------------------------------------------------------------------------------------ 64 bits


def _round8(v):
    """float64 values of at most 448 in magnitude, rounded to e4m3 (three bits after the leading one, 2^-9 steps at
    the least), ties to even."""
    step = torch.ldexp(torch.ones_like(v), (torch.frexp(v)[1].clamp(min=-5) - 4).to(torch.int32))
    return torch.round(v / step) * step


def _exact_blocks(z):
    """(code values, scales) of float64 rows in blocks of 1 x 128, by logarithms; every value is finite."""
    R, K = z.shape
    blocks = torch.zeros((R, _pad(K, BLOCK)), dtype=torch.float64, device=DEV)
    blocks[:, :K] = z
    blocks = blocks.view(R, -1, BLOCK)
    scale = torch.exp2(torch.ceil(torch.log2(blocks.abs().amax(dim=2) / 448)).clamp(min=-126))
    q = _round8(blocks / scale[..., None])
    padded = torch.full((R, _pad(scale.shape[1], 4)), 2.0 ** -126, dtype=torch.float64, device=DEV)
    padded[:, :scale.shape[1]] = scale
    return q.view(R, -1), padded


def _exact_values(q, scale, rows, n, k):
    """float64 values of an n x k matrix of codes."""
    e = torch.exp2(scale.view(torch.uint8).to(torch.float64) - 127)
    col = torch.arange(k, device=DEV) // BLOCK
    return q[:n, :k].to(torch.float64) * e[torch.arange(n, device=DEV) // rows][:, col]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"].double()
        if case["residual"]:
            x = x + s["r"].double()
        z = x / torch.sqrt((x ** 2).sum(dim=1, keepdim=True) / case["H"] + EPS) * s["gamma"].double()
        q, scale = _exact_blocks(z)
        out = {"q": q, "scale": scale}
        if case["residual"]:
            out["sum"] = x
        if case["normed"]:
            out["normed"] = z
        return out
    if case["op"] == "route":
        return _exact_route(case, s)
    if case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        y = torch.matmul(_exact_values(s["a"], s["sa"], 1, M, K), _exact_values(s["w"], s["sw"], BLOCK, N, K).t())
        if case["bias"]:
            y += s["b"].double()
        return torch.where(y < 0, 0.0, y) if case["relu"] else y
    T, H, F, E, k = (case[x] for x in ("T", "H", "F", "E", "k"))
    x = _exact_values(s["a"], s["sa"], 1, T, H)
    out = s["r"].double() if case["residual"] else torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for e in range(E):
        token, j = (s["ids"] == e).nonzero(as_tuple=True)
        if token.numel() == 0:
            continue
        gate = x[token] @ _exact_values(s["w_in"][e, 0], s["sw_in"][e, 0], BLOCK, F, H).t()
        up = x[token] @ _exact_values(s["w_in"][e, 1], s["sw_in"][e, 1], BLOCK, F, H).t()
        q, scale = _exact_blocks(gate * torch.sigmoid(gate) * up)
        p = (q.view(len(token), -1, BLOCK) * scale[:, :q.shape[1] // BLOCK, None]).flatten(1)[:, :F]
        o = p @ _exact_values(s["w_out"][e], s["sw_out"][e], BLOCK, H, F).t()
        out.index_add_(0, token, o * s["weight"][token, j].double()[:, None])
    return out


def _exact_route(case, s):
    l = s["logits"].double()
    T, E, k = case["T"], case["E"], case["k"]
    dead = torch.isinf(l)
    score = torch.softmax(l, dim=1).nan_to_num(0.0) if case["score"] == "softmax" else torch.sigmoid(l)
    choice = (score + s["b"].double() if case["bias"] else score).masked_fill(dead, -math.inf)
    if case["groups"] > 1:
        parts = choice.view(T, case["groups"], -1).clone()
        value = torch.zeros((T, case["groups"]), dtype=torch.float64, device=DEV)
        for b in range(min(case["best"], parts.shape[2])):
            top = parts.max(dim=2)
            value += top.values if b == 0 else top.values.nan_to_num(neginf=0.0)
            parts.scatter_(2, top.indices[..., None], -math.inf)
        open_ = torch.zeros_like(value, dtype=torch.bool)
        for _ in range(case["kept"]):
            at = _first_best(value)
            open_.scatter_(1, at, True)
            value.scatter_(1, at, -math.inf)
        choice = choice.masked_fill(~open_.repeat_interleave(E // case["groups"], dim=1), -math.inf)
    ids, weight = [], []
    for _ in range(k):
        at = _first_best(choice)
        none = torch.isneginf(choice.gather(1, at))
        ids.append(torch.where(none, -1, at))
        weight.append(torch.where(none, 0.0, score.gather(1, at)))
        choice.scatter_(1, at, -math.inf)
    ids, weight = torch.cat(ids, 1).to(torch.int32), torch.cat(weight, 1)
    weight = weight / weight.sum(dim=1, keepdim=True).clamp(min=1e-300)
    flat = ids.reshape(-1).cpu()
    groups = [(flat == e).nonzero()[:, 0] for e in range(E)]
    order = torch.cat(groups).to(torch.int32)
    order = torch.cat([order, torch.full((flat.numel() - order.numel(),), -1, dtype=torch.int32)])
    offsets = torch.tensor([0] + [len(x) for x in groups]).cumsum(0).to(torch.int32)
    return {"ids": ids, "weight": weight, "offsets": offsets, "order": order}


def _first_best(v):
    """The lowest index of each row's largest value, as a column."""
    n = v.shape[1]
    index = torch.arange(n, device=v.device).expand_as(v)
    return torch.where(v == v.amax(dim=1, keepdim=True), index, n).amin(dim=1, keepdim=True)

"""Performance cases of the operators that generate tokens with a layer of experts.

``groups``   a matrix rounded to 4 bits with a scale for each group of 32 columns, and the values it then stands for
``product``  the products of a few dense rows with a matrix of 4 bits: a projection, or the logits of a vocabulary
``layer``    a whole layer of experts for a few tokens: norm, router, the chosen experts' networks, and their sum
``sample``   the next token of each row of logits: temperature, top-k, top-p, min-p and one uniform number

Each case is one call a program makes for every token that it generates (``groups``: once for a weight).  ``listed()``
holds the named cases, ``draw()`` gives further ones of the same ranges, ``prepare()`` makes the inputs on the GPU from a
seed, ``run()`` is one call (in plain torch, or the library's where ``own`` is set), ``exact()`` the same result in 64 bits.

4-bit format: codes are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the lower columns in the
lower bits, one row padded with zeros to a multiple of 128 columns; a group's scale is a power of two, held as its exponent
(e8m0), the least one (2^-126 at least) that brings the group's largest magnitude to 6 or less; codes are rounded to
nearest even.  The experts' weights are e4m3 codes in blocks of 128 x 128 with such scales (448 in the place of 6), and
the rows that meet them are rounded to e4m3 in blocks of 1 x 128.
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GROUP = 32
BLOCK = 128
EPS = 1e-6


def listed():
    return [
        # A small weight of single precision whose width ends inside a group.
        dict(name="groups-odd", op="groups", R=777, K=1001, dtype="f32"),
        # A large projection's weight: memory bandwidth.
        dict(name="groups-weight", op="groups", R=16384, K=4096, dtype="bf16"),
        # One token through a square projection: latency.
        dict(name="product-token", op="product", M=1, N=4096, K=4096, dtype="bf16", out="bf16", bias=False, relu=False),
        # A few rows of an MLP whose widths are multiples of nothing, in single precision.
        dict(name="product-odd", op="product", M=7, N=2999, K=1001, dtype="f32", out="f32", bias=True, relu=True),
        # One token's logits over a vocabulary: the weights' bytes.
        dict(name="product-head", op="product", M=1, N=131072, K=4096, dtype="bf16", out="f32", bias=False, relu=False),
        # A full batch of generating sequences through a wide layer.
        dict(name="product-batch", op="product", M=64, N=16384, K=4096, dtype="bf16", out="bf16", bias=False,
             relu=False),
        # One token through its 8 of 64 experts: the chosen weights' bytes.
        dict(name="layer-token", op="layer", T=1, H=4096, F=1024, E=64, k=8, dtype="bf16", router="bf16",
             residual=True, score="softmax", bias=False, groups=1, kept=1, best=1, idle=0.0),
        # An odd batch with idle places, a balance bias, groups of experts, and widths that end inside a block.
        dict(name="layer-odd", op="layer", T=5, H=2001, F=701, E=24, k=3, dtype="f32", router="f32", residual=False,
             score="sigmoid", bias=True, groups=4, kept=2, best=2, idle=0.2),
        # As many tokens as the call takes: nearly every expert's weights.
        dict(name="layer-batch", op="layer", T=16, H=4096, F=1024, E=64, k=8, dtype="bf16", router="f32",
             residual=True, score="sigmoid", bias=True, groups=1, kept=1, best=1, idle=0.0),
        # One sequence's next token with every filter on: latency.
        dict(name="sample-token", op="sample", T=1, V=131072, dtype="f32", filters="all", banned=0.0),
        # An odd batch where each row has filters of its own, some rows none, some greedy, and some tokens are banned.
        dict(name="sample-odd", op="sample", T=37, V=50021, dtype="bf16", filters="mixed", banned=0.3),
        # A large batch over a large vocabulary.
        dict(name="sample-batch", op="sample", T=128, V=131072, dtype="f32", filters="mixed", banned=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of an operator, over its whole range of sizes, no dearer than the operator's largest listed one."""
    op = rng.choice(["groups", "product", "layer", "sample"])
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
    if op == "groups":
        return dict(op=op, R=_log(rng, 1, 131072), K=_log(rng, 1, 16384), dtype=dtype)
    if op == "product":
        return dict(op=op, M=_log(rng, 1, 64), N=_log(rng, 64, 131072), K=_log(rng, 64, 16384), dtype=dtype,
                    out=rng.choice(["f32", "bf16"]), bias=rng.random() < 0.5, relu=rng.random() < 0.5)
    if op == "sample":
        return dict(op=op, T=_log(rng, 1, 256), V=_log(rng, 2, 262144), dtype=dtype,
                    filters=rng.choice(["all", "mixed"]), banned=rng.choice([0.0, 0.3]))
    groups = rng.choice([1, 1, 2, 4, 8])
    E = groups * _log(rng, max(2, 4 // groups), 128 // groups)
    kept = rng.randint(1, groups)
    return dict(op=op, T=_log(rng, 1, 16), H=_log(rng, 256, 4096), F=_log(rng, 128, 2048), E=E,
                k=rng.randint(1, min(8, E // groups * kept)), dtype=dtype, router=rng.choice(["f32", "bf16"]),
                residual=rng.random() < 0.5, score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                groups=groups, kept=kept, best=rng.randint(1, 2), idle=rng.choice([0.0, 0.2]))


def _size(kind):
    return 4 if kind == "f32" else 2


def work(case):
    op = case["op"]
    if op == "groups":
        cells = case["R"] * case["K"]
        # read, written as 4 bits, read back, written as values of the same type
        return {"bytes": cells * (2 * _size(case["dtype"]) + 2 * (0.5 + 1 / GROUP)), "flops": 4 * cells}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K * (0.5 + 1 / GROUP) + M * K * _size(case["dtype"]) + M * N * _size(case["out"])
                + 4 * N * case["bias"], "flops": 2 * M * N * K}
    if op == "sample":
        cells = case["T"] * case["V"]
        return {"bytes": cells * _size(case["dtype"]) + 32 * case["T"], "flops": 20 * cells}
    T, H, F, E, k = (case[x] for x in ("T", "H", "F", "E", "k"))
    live = T * (1 - case["idle"])
    busy = E * (1 - (1 - k / E) ** live)  # experts that an even router reaches
    return {"bytes": busy * 3 * F * H + E * H * _size(case["router"]) + T * H * _size(case["dtype"])
            * (2 + case["residual"]) + 4 * H + 8 * T * k, "flops": 2 * T * E * H + 6 * live * k * F * H}


# ------------------------------------------------------------------------------------------------ inputs


def _pad(n, to):
    return -(-n // to) * to


def _powers(codes):
    """The powers of two that e8m0 codes (1 to 254) stand for."""
    return (codes.view(torch.uint8).to(torch.int32) << 23).view(torch.float32)


def _scale_codes(size, most_bits, exponent):
    """e8m0 codes of float32 maxima: the least scale that brings them to (1 + most_bits / 2^23) 2^exponent or less."""
    bits = size.view(torch.int32)
    return ((bits >> 23) - exponent + ((bits & 0x7FFFFF) > most_bits)).clamp(min=1)


def _quantize8(z, rows):
    """(codes, scale) of a (..., R, K) float32 tensor in blocks of rows x 128."""
    R, K = z.shape[-2:]
    z = torch.nn.functional.pad(z, (0, _pad(K, BLOCK) - K, 0, _pad(R, rows) - R))
    tiles = z.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, rows))  # (..., R/rows, rows, K/128, 128)
    code = _scale_codes(tiles.abs().amax(dim=(-3, -1)), 0x600000, 8)
    inverse = ((254 - code) << 23).view(torch.float32)[..., :, None, :, None]
    q = (tiles * inverse).flatten(-4, -3).flatten(-2)[..., :R, :].to(torch.float8_e4m3fn)
    scale = torch.nn.functional.pad(code.to(torch.uint8), (0, _pad(code.shape[-1], 4) - code.shape[-1]), value=1)
    return q.contiguous(), scale.contiguous().view(torch.float8_e8m0fnu)


def _values8(q, scale, rows):
    """The float32 values that (..., R, pitch) codes in blocks of rows x 128 stand for."""
    s = _powers(scale)[..., :q.shape[-1] // BLOCK]
    s = s.repeat_interleave(rows, dim=-2)[..., :q.shape[-2], :]
    return (q.to(torch.float32).unflatten(-1, (-1, BLOCK)) * s[..., None]).flatten(-2)


def _steps(v, bits, least):
    """float64 values rounded to `bits` bits after the leading one, in steps of 2^least at the least, ties to even."""
    step = torch.ldexp(torch.ones_like(v), (torch.frexp(v)[1] - 1 - bits).clamp(min=least).to(torch.int32))
    return torch.round(v / step) * step


def _rounded8(z):
    """The values of float64 rows rounded to 8 bits in blocks of 1 x 128, in float64."""
    T, K = z.shape
    blocks = torch.nn.functional.pad(z, (0, _pad(K, BLOCK) - K)).view(T, -1, BLOCK)
    # the maximum is compared with 448 times a power of two: a float holds every bit that decides it, rounded upwards
    size = blocks.abs().amax(dim=2)
    near = size.to(torch.float32)
    near = torch.where(near.double() < size, torch.nextafter(near, torch.full_like(near, math.inf)), near)
    scale = _powers(_scale_codes(near, 0x600000, 8).to(torch.uint8)).double()[..., None]
    return (_steps(blocks / scale, 3, -9) * scale).view(T, -1)[:, :K]


def _groups(x):
    """(values in units of the scale, scale codes) of a float32 matrix in groups of 32 columns."""
    R, K = x.shape
    tiles = torch.nn.functional.pad(x, (0, _pad(K, BLOCK) - K)).view(R, -1, GROUP)
    code = _scale_codes(tiles.abs().amax(dim=2), 0x400000, 2)
    scaled = tiles * ((254 - code) << 23).view(torch.float32)[..., None]
    a = scaled.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.round(a / step) * step * torch.sign(scaled), code.to(torch.uint8)


def _packed(v):
    """e2m1 codes, two to a byte, of (R, groups, 32) values that are all among the eight magnitudes."""
    a = v.abs()
    index = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    index = (index | torch.where(v < 0, 8, 0).to(torch.uint8)).flatten(1)
    return (index[:, 0::2] | (index[:, 1::2] << 4)).contiguous().view(torch.float4_e2m1fn_x2)


def _values4(codes, scales):
    """The float32 values of a 4-bit matrix, padding columns and all."""
    b = codes.view(torch.uint8)
    index = torch.stack([b & 15, b >> 4], dim=-1).flatten(1).to(torch.int64)
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0],
                         device=DEV)
    return (table[index].unflatten(1, (-1, GROUP)) * _powers(scales)[..., None]).flatten(1)


def _hidden(g, T, H):
    """Hidden states: normal, with a few columns ten times as wide, as trained models have them."""
    x = torch.randn((T, H), generator=g, device=DEV)
    return x * torch.where(torch.rand(H, generator=g, device=DEV) < 0.01, 10.0, 1.0)


def _experts_weights(g, shape):
    return _quantize8(torch.randn(shape, generator=g, device=DEV) / math.sqrt(shape[-1]), BLOCK)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)
    s = dict(case)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "groups":
        s["x"] = (torch.randn((case["R"], case["K"]), generator=g, device=DEV) / math.sqrt(case["K"])).to(dtype)
    elif case["op"] == "product":
        N, K = case["N"], case["K"]
        s["x"] = _hidden(g, case["M"], K).to(dtype)
        v, scale = _groups(torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K))
        s["w"], s["sw"] = _packed(v), scale.contiguous().view(torch.float8_e8m0fnu)
        s["b"] = 0.1 * torch.randn(N, generator=g, device=DEV) if case["bias"] else None
    elif case["op"] == "layer":
        T, H, F, E = (case[x] for x in ("T", "H", "F", "E"))
        s["x"] = _hidden(g, T, H).to(dtype)
        s["r"] = _hidden(g, T, H).to(dtype) if case["residual"] else None
        s["gamma"] = 1 + 0.1 * torch.randn(H, generator=g, device=DEV)
        s["wr"] = (torch.randn((E, H), generator=g, device=DEV) / math.sqrt(H)).to(DTYPES[case["router"]])
        # a balance bias moves in steps of a thousandth
        steps = torch.randint(-100, 101, (E,), generator=g, device=DEV)
        s["b"] = steps.to(torch.float32) * 1e-3 if case["bias"] else None
        s["live"] = torch.rand(T, generator=g, device=DEV) >= case["idle"] if case["idle"] > 0 else None
        s["w_in"], s["sw_in"] = _experts_weights(g, (E, 2, F, H))
        s["w_out"], s["sw_out"] = _experts_weights(g, (E, H, F))
    else:
        T, V = case["T"], case["V"]
        # A model's logits: a broad bulk and a few tokens well above it.
        l = 2 * torch.randn((T, V), generator=g, device=DEV)
        l = l + 8 * torch.rand((T, 1), generator=g, device=DEV) * (torch.rand((T, V), generator=g, device=DEV) < 1e-4)
        if case["banned"] > 0:
            l = torch.where(torch.rand((T, V), generator=g, device=DEV) < case["banned"], -math.inf, l)
        s["logits"] = l.to(dtype)
        s["u"] = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
        # Rows of sequences with settings of their own; where they are mixed, each is off for a share of the rows.
        off = torch.rand((4, T), generator=g, device=DEV) < (0.3 if case["filters"] == "mixed" else 0.0)
        between = torch.rand((4, T), generator=g, device=DEV)
        s["temperature"] = torch.where(off[0], torch.where(between[0] < 0.5, 0.0, 1.0), 0.5 + between[0])
        s["top_k"] = torch.where(off[1], 0, 1 + (200 * between[1]).to(torch.int32)).to(torch.int32)
        s["top_p"] = torch.where(off[2], 1.0, 0.7 + 0.29 * between[2])
        s["min_p"] = torch.where(off[3], 0.0, 0.1 * between[3])
    return s


# ------------------------------------------------------------------------------------------------ one call


def run(s):
    return (_own if own else _plain)[s["op"]](s)


def _plain_groups(s):
    v, code = _groups(s["x"].to(torch.float32))
    values = (v * _powers(code)[..., None]).flatten(1)[:, :s["K"]].to(s["x"].dtype)
    return {"values": values, "scale": code.view(torch.float8_e8m0fnu)}


def _plain_product(s):
    y = s["x"].to(torch.float32) @ _values4(s["w"], s["sw"])[:, :s["K"]].t()
    if s["b"] is not None:
        y = y + s["b"]
    if s["relu"]:
        y = y.clamp(min=0)
    return y.to(DTYPES[s["out"]])


def _plain_choice(l, s):
    """(ids, weight) of each row of float64 logits; an idle row's are all -inf."""
    T, E = l.shape
    there = l > -math.inf
    if s["score"] == "softmax":
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
    return torch.where(chosen, ids, -1).to(torch.int32), weight


def _plain_layer(s):
    T, H, F, E, k = (s[x] for x in ("T", "H", "F", "E", "k"))
    # The norm and the router's logits are held in 64 bits: which experts are chosen, and how rows are rounded to 8 bits,
    # is then the same whatever the order of a sum.
    x = s["x"].to(torch.float64)
    if s["r"] is not None:
        x = x + s["r"].to(torch.float64)
    z = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS) * s["gamma"].to(torch.float64)
    l = z @ s["wr"].to(torch.float64).t()
    if s["live"] is not None:
        l = torch.where(s["live"][:, None], l, -math.inf)
    ids, weight = _plain_choice(l, s)
    a = _rounded8(z).to(torch.float32)
    flat = ids.reshape(-1).long()
    w_in, sw_in, w_out, sw_out = s["w_in"], s["sw_in"], s["w_out"], s["sw_out"]
    if T * k <= E:  # few slots: each takes its own expert's weights
        at, lanes = flat.clamp(min=0), torch.arange(T * k, device=DEV)[:, None]
        w_in, w_out = w_in.view(torch.uint8)[at].view(w_in.dtype), w_out.view(torch.uint8)[at].view(w_out.dtype)
        sw_in, sw_out = sw_in.view(torch.uint8)[at], sw_out.view(torch.uint8)[at]
        there = (flat >= 0)[:, None]
    else:  # every expert has a place for every token
        hit = flat.view(T, k)[None] == torch.arange(E, device=DEV)[:, None, None]  # (E, T, k)
        there = hit.any(dim=2)
        lanes = torch.arange(T, device=DEV) * k + hit.to(torch.uint8).argmax(dim=2)
    rows = torch.where(there[..., None], a[lanes // k], 0.0).transpose(1, 2).contiguous()
    z = torch.bmm(_values8(w_in, sw_in, BLOCK).flatten(1, 2)[..., :H].contiguous(), rows)  # (experts, 2 F, lanes)
    gate, up = z[:, :F], z[:, F:]
    p = gate / (1 + torch.exp(-gate)) * up
    lines = p.transpose(1, 2).reshape(-1, F).to(torch.float64)
    p = _rounded8(lines).to(torch.float32).view(p.shape[0], -1, F).transpose(1, 2).contiguous()
    o = torch.bmm(_values8(w_out, sw_out, BLOCK)[..., :F].contiguous(), p).transpose(1, 2)  # (experts, lanes, H)
    part = torch.zeros((T * k + 1, H), device=DEV)
    share = torch.where(there, weight.reshape(-1)[lanes], 0.0)
    part[torch.where(there, lanes, T * k)] = o * share[..., None]
    out = x.to(torch.float32) + part[:T * k].view(T, k, H).sum(dim=1)
    return {"out": out.to(s["x"].dtype), "ids": ids, "weight": weight}


def _plain_sample(s):
    # Tokens are kept and drawn by sums in 64 bits: 32 do not tell the tokens of a large vocabulary apart.
    T, V = s["T"], s["V"]
    l = s["logits"].to(torch.float64)
    there = l > -math.inf
    l, order = torch.sort(torch.where(there, l, -math.inf), dim=1, descending=True, stable=True)
    there = l > -math.inf
    greedy = (s["temperature"] <= 0)[:, None]
    x = (l - l[:, :1]) / torch.where(greedy, 1.0, s["temperature"].to(torch.float64)[:, None])
    p = torch.where(there, torch.exp(x), 0.0)
    place = torch.arange(V, device=DEV)[None]
    k = s["top_k"].to(torch.int64)[:, None]
    keep = there & ((k <= 0) | (place < k)) & (~greedy | (place == 0))
    p = torch.where(keep, p, 0.0)
    sums = p.cumsum(dim=1)
    share = s["top_p"].to(torch.float64)[:, None]
    first = sums - p < share * sums[:, -1:]  # what comes before has not reached the share
    least = torch.log(s["min_p"].to(torch.float64))[:, None]
    keep = keep & ((share >= 1) | first) & (x >= least)
    p = torch.where(keep, p, 0.0)
    total = p.sum(dim=1, keepdim=True)
    mass = torch.zeros_like(p).scatter_(1, order, p)
    sums = mass.cumsum(dim=1)
    hit = (sums > s["u"][:, None] * total) & (mass > 0)
    ids = torch.where(hit.any(dim=1), hit.to(torch.uint8).argmax(dim=1), -1)
    prob = mass.gather(1, ids.clamp(min=0)[:, None]) / total
    prob = torch.where(ids >= 0, prob[:, 0], 0.0).to(torch.float32)
    return {"ids": ids.to(torch.int32), "prob": prob, "kept": keep.sum(dim=1).to(torch.int32)}


_plain = {"groups": _plain_groups, "product": _plain_product, "layer": _plain_layer, "sample": _plain_sample}


def _own_groups(s):
    import paper_1708_02937_amd as sd

    codes, scale = sd.quantize_groups(s["x"])
    return {"values": sd.widen_groups(codes, scale, s["K"], dtype=s["x"].dtype), "scale": scale}


def _own_product(s):
    import paper_1708_02937_amd as sd

    return sd.product_groups(s["x"], s["w"], s["sw"], bias=s["b"], ymax=math.inf if s["relu"] else None,
                             dtype=DTYPES[s["out"]])


def _own_layer(s):
    import paper_1708_02937_amd as sd

    out, ids, weight = sd.experts_layer(s["x"], s["gamma"], s["wr"], s["k"], s["w_in"], s["sw_in"], s["w_out"],
                                        s["sw_out"], s["F"], eps=EPS, residual=s["r"], live=s["live"],
                                        score=s["score"], bias=s["b"], groups=s["groups"], groups_kept=s["kept"],
                                        group_best=s["best"])
    return {"out": out, "ids": ids, "weight": weight}


def _own_sample(s):
    import paper_1708_02937_amd as sd

    ids, prob, kept = sd.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                                top_p=s["top_p"], min_p=s["min_p"])
    return {"ids": ids, "prob": prob, "kept": kept}


_own = {"groups": _own_groups, "product": _own_product, "layer": _own_layer, "sample": _own_sample}


# ------------------------------------------------------------------------------------------------ 64 bits


MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_values4(codes, scales, k):
    """float64 values of an n x k 4-bit matrix, code by code."""
    b = codes.view(torch.uint8)
    v = torch.zeros((b.shape[0], 2 * b.shape[1]), dtype=torch.float64, device=DEV)
    for half in (0, 1):
        code = (b if half == 0 else b >> 4) & 15
        for i, m in enumerate(MAGNITUDES):
            v[:, half::2] += m * ((code == i).double() - (code == i + 8).double())
    e = torch.exp2(scales.view(torch.uint8).double() - 127)
    return (v * e[:, torch.arange(v.shape[1], device=DEV) // GROUP])[:, :k]


def _exact_values8(q, scale, n, k):
    """float64 values of an n x k matrix of e4m3 codes in blocks of 128 x 128."""
    e = torch.exp2(scale.view(torch.uint8).double() - 127)
    at = torch.arange(n, device=DEV) // BLOCK, torch.arange(k, device=DEV) // BLOCK
    return q[:n, :k].double() * e[at[0]][:, at[1]]


def _exact_round8(z):
    """float64 rows rounded to 8 bits in blocks of 1 x 128, the scales by logarithms and a comparison."""
    R, K = z.shape
    out = torch.empty_like(z)
    for c in range(0, K, BLOCK):
        v = z[:, c:c + BLOCK]
        big = v.abs().amax(dim=1, keepdim=True)
        e = torch.floor(torch.log2(torch.where(big > 0, big, 1e-300) / 448)).clamp(min=-126)
        e = torch.where(big > 448 * torch.exp2(e), e + 1, e)
        v = v / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, c:c + BLOCK] = torch.round(v / step) * step * torch.exp2(e)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "groups":
        x, K = s["x"].double(), case["K"]
        out = torch.zeros((case["R"], _pad(K, BLOCK)), dtype=torch.float64, device=DEV)
        scale = torch.full((case["R"], _pad(K, BLOCK) // GROUP), 2.0 ** -126, dtype=torch.float64, device=DEV)
        for c in range(0, K, GROUP):
            v = x[:, c:c + GROUP]
            big = v.abs().amax(dim=1, keepdim=True)
            e = torch.floor(torch.log2(torch.where(big > 0, big, 1e-300) / 6)).clamp(min=-126)
            e = torch.where(big > 6 * torch.exp2(e), e + 1, e)
            scale[:, c // GROUP] = torch.exp2(e)[:, 0]
            a = v.abs() / torch.exp2(e)
            r = torch.zeros_like(a)
            for i in range(7):  # a value stands past the middle of two magnitudes, or on it and goes to the even one
                half = (MAGNITUDES[i] + MAGNITUDES[i + 1]) / 2
                r = torch.where((a > half) | ((a == half) & (i % 2 == 1)), MAGNITUDES[i + 1], r)
            out[:, c:c + v.shape[1]] = torch.where(v < 0, -r, r) * torch.exp2(e)
        return {"values": out[:, :K], "scale": scale}
    if case["op"] == "product":
        N, K = case["N"], case["K"]
        x, parts = s["x"].double().t().contiguous(), []
        for n in range(0, N, 8192):
            parts.append(torch.matmul(_exact_values4(s["w"][n:n + 8192], s["sw"][n:n + 8192], K), x).t())
        y = torch.cat(parts, dim=1)
        if case["bias"]:
            y = y + s["b"].double()
        return torch.where(y < 0, 0.0, y) if case["relu"] else y
    return _exact_sample(case, s) if case["op"] == "sample" else _exact_layer(case, s)


def _exact_layer(case, s):
    T, H, F, E, k = (case[x] for x in ("T", "H", "F", "E", "k"))
    x = s["x"].double() + (s["r"].double() if case["residual"] else 0.0)
    z = x / torch.sqrt((x ** 2).sum(dim=1, keepdim=True) / H + EPS) * s["gamma"].double()
    logits = torch.stack([(z * s["wr"][e].double()).sum(dim=1) for e in range(E)], dim=1).cpu()
    live = [True] * T if s["live"] is None else s["live"].tolist()
    bias = [0.0] * E if s["b"] is None else s["b"].double().tolist()
    a, out, size = _exact_round8(z), x.clone(), E // case["groups"]
    ids, weight = torch.full((T, k), -1, dtype=torch.int32), torch.zeros((T, k), dtype=torch.float64)
    for t in range(T):
        if not live[t]:
            continue
        score = (torch.softmax(logits[t], 0) if case["score"] == "softmax" else torch.sigmoid(logits[t])).tolist()
        choice = [score[e] + bias[e] for e in range(E)]
        worth = [sum(sorted(choice[g * size:(g + 1) * size], reverse=True)[:case["best"]])
                 for g in range(case["groups"])]
        stay = sorted(range(case["groups"]), key=lambda g: (-worth[g], g))[:case["kept"]]
        pick = sorted((e for e in range(E) if e // size in stay), key=lambda e: (-choice[e], e))[:k]
        total = sum(score[e] for e in pick)
        for j, e in enumerate(pick):
            ids[t, j], weight[t, j] = e, score[e] / total
    for e in range(E):
        token, j = (ids == e).nonzero(as_tuple=True)
        if token.numel() == 0:
            continue
        rows = a[token.to(DEV)]
        gate = rows @ _exact_values8(s["w_in"][e, 0], s["sw_in"][e, 0], F, H).t()
        up = rows @ _exact_values8(s["w_in"][e, 1], s["sw_in"][e, 1], F, H).t()
        o = _exact_round8(gate * torch.sigmoid(gate) * up) @ _exact_values8(s["w_out"][e], s["sw_out"][e], H, F).t()
        out.index_add_(0, token.to(DEV), o * weight[token, j].to(DEV)[:, None])
    return {"out": out, "ids": ids, "weight": weight}


def _exact_sample(case, s):
    import numpy as np

    T, V = case["T"], case["V"]
    logits = s["logits"].float().cpu().numpy().astype(np.float64)
    u, temperature, top_k, top_p, min_p = (s[x].double().cpu().numpy()
                                           for x in ("u", "temperature", "top_k", "top_p", "min_p"))
    ids, prob, count = np.full(T, -1, np.int32), np.zeros(T), np.zeros(T, np.int32)
    for t in range(T):
        order = np.lexsort((np.arange(V), -logits[t]))
        order = order[np.isfinite(logits[t][order])]
        if not len(order):
            continue
        if temperature[t] <= 0:
            order = order[:1]
        elif top_k[t] > 0:
            order = order[:int(top_k[t])]
        p = np.exp((logits[t][order] - logits[t][order[0]]) / (temperature[t] if temperature[t] > 0 else 1.0))
        keep = len(p)
        if top_p[t] < 1:
            keep = 1 + int(np.searchsorted(np.cumsum(p), top_p[t] * np.sum(p)))
        p = p[:keep]
        p = p[p >= min_p[t]]
        order = np.sort(order[:len(p)])
        mass = np.exp((logits[t][order] - logits[t].max()) / (temperature[t] if temperature[t] > 0 else 1.0))
        at = min(int(np.searchsorted(np.cumsum(mass), u[t] * mass.sum(), side="right")), len(order) - 1)
        ids[t], prob[t], count[t] = order[at], mass[at] / mass.sum(), len(order)
    return {"ids": torch.from_numpy(ids), "prob": torch.from_numpy(prob), "kept": torch.from_numpy(count)}

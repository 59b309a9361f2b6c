"""Plain 64-bit definitions of the operators of a layer of experts, on the CPU (no code of the library)."""

import numpy as np

BLOCK = 128


def pad(n, to):
    return -(-n // to) * to


def e4m3_table():
    """The value of each of the 256 codes."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c > 127, -v, v)


TABLE = e4m3_table()
_POSITIVE = TABLE[:127]  # 0 to 448, ascending


def encode(v):
    """Codes of float64 values of at most 448 in magnitude: nearest, ties to the even code; NaN for what is not finite."""
    a = np.abs(np.where(np.isfinite(v), v, 0.0))
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(np.isfinite(v), code, 127)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quantize(z, block_rows=1):
    """(codes, scale codes) of one rows x k matrix; the scale by search, not by arithmetic on exponents."""
    z = np.asarray(z, dtype=np.float64)
    rows, k = z.shape
    blocks, sp = -(-k // BLOCK), pad(-(-k // BLOCK), 4)
    sr = -(-rows // block_rows)
    codes = np.zeros((rows, blocks * BLOCK), np.uint8)
    scales = np.full((sr, sp), 1, np.uint8)
    for r in range(sr):
        for b in range(blocks):
            t = z[r * block_rows:(r + 1) * block_rows, b * BLOCK:(b + 1) * BLOCK]
            big = np.max(np.abs(t[np.isfinite(t)]), initial=0.0)
            e = -126
            if big > 0:
                e = max(-126, int(np.ceil(np.log2(big / 448))) - 1)
                while big * 2.0 ** -e > 448:
                    e += 1
            codes[r * block_rows:(r + 1) * block_rows, b * BLOCK:b * BLOCK + t.shape[1]] = encode(t * 2.0 ** -e)
            scales[r, b] = e + 127
    return codes, scales


def values(codes, scales, k, block_rows=1):
    """float64 values of a blocked matrix."""
    s = 2.0 ** (scales.astype(np.float64) - 127)
    s = np.repeat(s, block_rows, axis=0)[:codes.shape[0]]
    return (TABLE[codes] * np.repeat(s, BLOCK, axis=1)[:, :codes.shape[1]])[:, :k]


def round_bf16(a):
    """float64 values rounded once to bfloat16 (8 significant bits, ties to even); normal range only."""
    m, e = np.frexp(a)  # 0.5 <= |m| < 1
    with np.errstate(invalid="ignore"):
        return np.where(np.isfinite(a), np.ldexp(np.rint(m * 256), e - 8), a)


def norm(x, gamma, eps, residual=None):
    s = x.astype(np.float64)
    if residual is not None:
        s = s + residual.astype(np.float64)
    with np.errstate(invalid="ignore"):
        return s, s / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps) * gamma.astype(np.float64)


def route(logits, k, score, bias, groups, kept, best, normalize, factor):
    """(ids, weight in float64) token by token, by sorting (choice descending, index ascending)."""
    T, E = logits.shape
    ids, weight = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        l = logits[t].astype(np.float64)
        there = l > -np.inf  # False for NaN
        if not there.any():
            continue
        if score == "sigmoid":
            s = 1 / (1 + np.exp(-l))
        elif (l == np.inf).any():
            s = (l == np.inf) / np.sum(l == np.inf)
        else:
            s = np.where(there, np.exp(np.where(there, l, 0) - l[there].max()), 0.0)
            s = s / s.sum()
        c = np.where(there, s if bias is None else s + bias.astype(np.float64), -np.inf)
        c = np.where(np.isnan(c), -np.inf, c)
        if groups > 1:
            size = E // groups
            worth = []
            for g in range(groups):
                top = np.sort(c[g * size:(g + 1) * size])[::-1][:best]
                worth.append(np.sum(top[top > -np.inf]) if top[0] > -np.inf else -np.inf)
            stay = sorted(range(groups), key=lambda g: (-worth[g], g))[:kept]
            c = np.where(np.isin(np.arange(E) // size, stay), c, -np.inf)
        pick = [e for e in sorted(range(E), key=lambda e: (-c[e], e)) if c[e] > -np.inf][:k]
        total = sum(s[e] for e in pick) if normalize else 1.0
        for j, e in enumerate(pick):
            ids[t, j] = e
            weight[t, j] = s[e] / total * factor if total > 0 else 0.0
    return ids, weight


def plan(ids, E):
    flat = ids.reshape(-1)
    lists = [np.flatnonzero(flat == e) for e in range(E)]
    offsets = np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)
    order = np.full(flat.size, -1, np.int32)
    order[:offsets[-1]] = np.concatenate(lists) if flat.size else []
    return offsets, order

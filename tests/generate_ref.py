"""Plain 64-bit definitions of the operators that generate tokens, on the CPU (no code of the library)."""

import numpy as np

from tests import blocks_ref as ref

GROUP = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TABLE = np.concatenate([MAGNITUDES, -MAGNITUDES])


def encode4(v):
    """Codes of float64 values of at most 6 in magnitude: nearest, ties to the even code."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(MAGNITUDES, a), 0, 7)
    lo = np.maximum(hi - 1, 0)
    up, down = MAGNITUDES[hi] - a, a - MAGNITUDES[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code | np.where(np.signbit(v), 8, 0)).astype(np.uint8)


def pack4(index):
    """Codes of rows x an even number of columns, two to a byte, the lower column in the lower bits."""
    return (index[:, 0::2] | index[:, 1::2] << 4).astype(np.uint8)


def quantize4(x):
    """(packed codes, scale codes) of one rows x k matrix; the scale by search."""
    with np.errstate(invalid="ignore"):
        x = np.asarray(x, dtype=np.float64)
    rows, k = x.shape
    cols = ref.pad(k, 128)
    z = np.zeros((rows, cols))
    z[:, :k] = x
    index, scales = np.zeros((rows, cols), np.uint8), np.ones((rows, cols // GROUP), np.uint8)
    for g in range(cols // GROUP):
        t = z[:, g * GROUP:(g + 1) * GROUP]
        for r in range(rows):
            big = np.max(np.abs(t[r]))
            if not np.isfinite(big):  # NaN too
                scales[r, g] = 255
                continue
            e = -126
            if big > 0:
                e = max(-126, int(np.ceil(np.log2(big / 6))) - 1)
                while big * 2.0 ** -e > 6:
                    e += 1
            index[r, g * GROUP:(g + 1) * GROUP] = encode4(t[r] * 2.0 ** -e)
            scales[r, g] = e + 127
    return pack4(index), scales


def values4(codes, scales, k):
    """float64 values of a 4-bit matrix."""
    index = np.empty((codes.shape[0], 2 * codes.shape[1]), np.int64)
    index[:, 0::2], index[:, 1::2] = codes & 15, codes >> 4
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (TABLE[index] * np.repeat(s, GROUP, axis=1))[:, :k]


def sample(l, u, temperature, top_k, top_p, min_p):
    """(index, share, kept, room) of one row of float64 logits, by sorting; room: how far, relative to all masses, the
    decisions are from being other ones (0 where a sum is exactly a share)."""
    order = np.lexsort((np.arange(l.size), -l))
    order = order[l[order] > -np.inf]  # NaN sorts last and is dropped
    if not order.size:
        return -1, 0.0, 0, 1.0
    if not temperature > 0:
        return int(order[0]), 1.0, 1, 1.0
    top = l[order[0]]
    with np.errstate(invalid="ignore"):
        x = np.where(l[order] == top, 0.0, (top - l[order]) / min(temperature, 1e300))
    p = np.exp(-x.astype(np.longdouble))
    k = top_k if 0 < top_k < order.size else order.size
    keep, room = k, 1.0
    if top_p < 1:
        sums = np.cumsum(p[:k])
        share = max(top_p, 0.0) * sums[-1]
        keep = 1 + int(np.searchsorted(sums, share))
        room = float(np.min(np.abs(sums - share)) / sums[-1])
    if min_p > 0:
        keep = min(keep, int(np.sum(x <= -np.log(min(min_p, 1.0)))))
    kept = np.sort(order[:keep])
    mass = np.zeros(l.size, np.longdouble)
    mass[order[:keep]] = p[:keep]
    sums = np.cumsum(mass[kept])
    at = min(int(np.searchsorted(sums, u * sums[-1], side="right")), kept.size - 1)
    while at > 0 and mass[kept[at]] == 0:
        at -= 1
    room = min(room, float(np.min(np.abs(sums - u * sums[-1])) / sums[-1]))
    return int(kept[at]), float(mass[kept[at]] / sums[-1]), keep, room

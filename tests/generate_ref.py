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

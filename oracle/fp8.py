"""Oracle of the paged cache in 8 bits (test infrastructure): e4m3 codes written
from the format's definition, and the write of a call's rows into pages with a scale
for each page and head, in 64 bits.
"""
import numpy as np

PAGE = 16
CODE_MAX, LEAST, MOST = 448.0, 2.0 ** -100, 2.0 ** 121


def _values():
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(c & 127) == 127] = np.nan
    return np.where(c & 128, -v, v)


VALUES = _values()  # of every code
_POSITIVE = VALUES[:127]


def decode(codes):
    return VALUES[codes]


def encode(x):
    """To nearest, ties to the even code; beyond 448 to 448, what is not finite to NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), CODE_MAX)
    hi = np.minimum(np.searchsorted(_POSITIVE, a), 126)
    lo = np.maximum(hi - 1, 0)
    up = _POSITIVE[hi] - a < a - _POSITIVE[lo]
    tie = _POSITIVE[hi] - a == a - _POSITIVE[lo]
    c = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
    c = np.where(_POSITIVE[hi] == a, hi, c).astype(np.uint8)
    return np.where(np.isfinite(x), c | np.where(np.signbit(x), 128, 0), 127).astype(np.uint8)


def runs(slots):
    """(first row, rows, page, offset) of every page's rows of a call."""
    t = 0
    while t < len(slots):
        n = 1
        if slots[t] >= 0:
            while t + n < len(slots) and slots[t + n] == slots[t] + n and (slots[t] + n) % PAGE:
                n += 1
            yield t, n, int(slots[t]) // PAGE, int(slots[t]) % PAGE
        t += n


def put(x, slots, codes, scale):
    """Rows x [T, H, D] to `slots` of codes [pages, 16, H, D] with scale [pages, H]:
    returns (values to hold / scale of their page before rounding, with the rows that
    were there as they are after; the codes as they should be; the scales)."""
    codes, scale = codes.copy(), scale.astype(np.float64).copy()
    exact = decode(codes)
    for t, n, page, off in runs(slots):
        rows = x[t: t + n].astype(np.float64)
        need = np.where(np.isfinite(rows), np.abs(rows), 0.0).max((0, 2)) / CODE_MAX
        for h in range(x.shape[1]):
            if off == 0:
                s = max(need[h], LEAST)
            else:
                s = scale[page, h]
                if not LEAST <= s <= MOST:
                    s = LEAST
                k = 0
                while need[h] > s * 2.0 ** k:
                    k += 1
                s *= 2.0 ** k
                if k:
                    codes[page, :off, h] = np.where(np.isnan(exact[page, :off, h]), codes[page, :off, h],
                                                    encode(exact[page, :off, h] * 2.0 ** -k))
                    exact[page, :off, h] = decode(codes[page, :off, h])
            scale[page, h] = s
            exact[page, off: off + n, h] = rows[:, h] / s
            codes[page, off: off + n, h] = encode(rows[:, h] / s)
    return exact, codes, scale

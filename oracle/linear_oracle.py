"""Plain 64-bit definitions of the 8-bit linear-layer operators (numpy).

Test infrastructure only; written from the definitions in include/muonbp.h.
"""

import numpy as np

BLOCK, GROUP, E_MIN = 128, 512, -110
# (exponent bits' bias, mantissa bits, largest value's exponent)
FORMATS = {0: (7, 3, 8), 1: (15, 2, 15)}  # e4m3, e5m2


def code_values(fmt):
    """The value of each of the 256 codes."""
    bias, mant, _ = FORMATS[fmt]
    out = np.empty(256)
    for code in range(256):
        sign = -1.0 if code & 128 else 1.0
        exp, frac = (code & 127) >> mant, code & ((1 << mant) - 1)
        if fmt == 0 and code & 127 == 127:
            v = np.nan  # e4m3: one NaN, no infinity
        elif fmt == 1 and exp == 31:
            v = np.inf if frac == 0 else np.nan
        elif exp == 0:
            v = frac * 2.0 ** (1 - bias - mant)
        else:
            v = (1 + frac / 2 ** mant) * 2.0 ** (exp - bias)
        out[code] = sign * v
    return out


def scale_exponent(amax, fmt):
    """The smallest e >= E_MIN with amax <= 2^e 1.75 2^top."""
    top = FORMATS[fmt][2]
    e = E_MIN
    if amax > 0:
        m, k = np.frexp(amax)  # amax = m 2^k, 1/2 <= m < 1
        e = max(E_MIN, int(k) - 1 - top + (1 if m > 0.875 else 0))
    return e


def nearest(v, fmt):
    """Codes of the nearest values of the type, ties to the even code; NaN and
    infinities as the type has them."""
    table = code_values(fmt)
    pos = table[:128]
    fin = np.where(np.isfinite(pos))[0]
    grid = pos[fin]
    a = np.abs(np.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0))
    hi = np.clip(np.searchsorted(grid, a), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - grid[lo], grid[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = fin[pick] | np.where(np.signbit(v), 128, 0)
    nan = 127
    code = np.where(np.isnan(v), nan, code)
    inf = 124 if fmt == 1 else nan
    return np.where(np.isinf(v), inf | np.where(np.signbit(v), 128, 0), code).astype(np.uint8)


def quantize(x, fmt=0, tile=False):
    """(codes rows x padded cols, biased exponents rows x blocks)."""
    r, c = x.shape
    nb = -(-c // BLOCK)
    pad = np.zeros((r, nb * BLOCK))
    pad[:, :c] = x
    fin = np.where(np.isfinite(pad), np.abs(pad), 0.0).reshape(r, nb, BLOCK).max(2, initial=0.0)
    if tile:
        for i in range(0, r, BLOCK):
            fin[i:i + BLOCK] = fin[i:i + BLOCK].max(0)
    e = np.array([[scale_exponent(v, fmt) for v in row] for row in fin], dtype=np.int64).reshape(r, nb)
    codes = nearest(pad / np.exp2(np.repeat(e, BLOCK, 1).astype(float)), fmt)
    return codes, e + 127


def words(e):
    """Scale words [ceil(blocks / 4)][rows] of biased exponents."""
    r, nb = e.shape
    p = np.zeros((r, -(-nb // 4) * 4), dtype=np.uint32)
    p[:, :nb] = e
    p = p.reshape(r, -1, 4)
    return (p[..., 0] | p[..., 1] << 8 | p[..., 2] << 16 | p[..., 3] << 24).T


def values(codes, e, cols, fmt=0):
    return (code_values(fmt)[codes] * np.exp2(np.repeat(e - 127, BLOCK, 1).astype(float)))[:, :cols]


def logistic(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def gated_forward(gate, up):
    return gate * logistic(gate) * up


def gated_backward(dh, gate, up):
    s = logistic(gate)
    return dh * up * s * (1 + gate * (1 - s)), dh * gate * s

"""Plain references of the block formats and the gated block, in 64 bits (NumPy)."""
import math

import numpy as np

FMTS = {(4, 3): 8, (5, 2): 8, (2, 1): 4}


def code_values(f):
    """The finite non-negative values of a narrow format, ascending: the index is the code."""
    wE, wF = f
    bias = 2 ** (wE - 1) - 1
    v = []
    for c in range(2 ** (wE + wF)):
        e, m = c >> wF, c & (2 ** wF - 1)
        v.append(math.ldexp(m, 1 - bias - wF) if e == 0 else math.ldexp(2 ** wF + m, e - bias - wF))
    if f == (4, 3):
        v = v[:-1]          # S.1111.111 is NaN
    if f == (5, 2):
        v = v[:-4]          # the highest exponent holds infinity and NaN
    return np.array(v)


def decode(codes, f):
    """The values of codes (integers), unscaled, float64."""
    wE, wF = f
    v = code_values(f)
    full = np.full(2 ** (wE + wF), np.nan)
    full[:len(v)] = v
    if f == (5, 2):
        full[len(v)] = np.inf
    codes = np.asarray(codes, dtype=np.int64)
    m = full[codes & (2 ** (wE + wF) - 1)]
    return np.where(codes >> (wE + wF), -m, m)


def limit(f):
    """(midpoint between the largest value and the step above it, whether it rounds up)."""
    v = code_values(f)
    return v[-1] + (v[-1] - v[-2]) / 2, len(v) % 2 == 0  # the step above would have an even code


def pow2_scale(amax, f):
    """The scale exponent of a group whose largest finite magnitude is amax."""
    lim, up = limit(f)
    k = -110
    if amax > 0:
        k = max(k, math.frexp(amax / lim)[1] - 3)
    while math.ldexp(amax, -k) > lim or (up and math.ldexp(amax, -k) == lim):
        k += 1
    return k


def nearest_codes(x, f):
    """Codes of scaled values: to nearest, ties to the even code; beyond the largest: the largest."""
    v = code_values(f)
    mid = (v[1:] + v[:-1]) / 2
    a = np.abs(x)
    i = np.searchsorted(mid, a, side="left")        # ties go down
    tie = (i < len(mid)) & (a == mid[np.minimum(i, len(mid) - 1)]) & (i % 2 == 1)
    i = i + tie
    nan_code = 2 ** sum(f) - 1
    if f == (4, 3):
        i = np.where(np.isfinite(x), i, nan_code)
    if f == (5, 2):
        i = np.where(np.isnan(x), nan_code, np.where(np.isinf(x), len(v), i))
    return i + (np.signbit(x).astype(np.int64) << sum(f))


def pack(x, f, group=32, scale="pow2"):
    """(codes [rows, cols], scale factors [rows, groups], scale exponents or None) of float64
    values that are float32 ones; scale: "pow2", or a function rounding a factor to its type."""
    rows, cols = x.shape
    groups = -(-cols // group)
    codes = np.zeros((rows, cols), dtype=np.int64)
    factors = np.zeros((rows, groups))
    for r in range(rows):
        for g in range(groups):
            v = x[r, g * group:(g + 1) * group]
            fin = np.abs(v[np.isfinite(v)])
            amax = float(fin.max()) if fin.size else 0.0
            if scale == "pow2":
                s = math.ldexp(1.0, pow2_scale(amax, f))
            else:
                s = float(scale(np.float32(amax) / np.float32(6)))
            if scale == "pow2":
                n = v / s
            else:   # the division is a float32 one
                with np.errstate(all="ignore"):
                    n = (v.astype(np.float32) / np.float32(s)).astype(np.float64) if s > 0 else v * 0
            if f == (2, 1) and fin.size < v.size:
                s = math.nan
                n = np.where(np.isfinite(v), n, 0.0)
            codes[r, g * group:(g + 1) * group] = nearest_codes(n, f)
            factors[r, g] = s
    return codes, factors


def unpack(codes, factors, f, group=32):
    with np.errstate(invalid="ignore", over="ignore"):
        return decode(codes, f) * np.repeat(factors, group, 1)[:, :codes.shape[1]]


def nibbles(packed, cols):
    """4-bit codes [rows, cols] of packed bytes."""
    both = np.stack([packed & 15, packed >> 4], 2).reshape(packed.shape[0], -1)
    return both[:, :cols].astype(np.int64)


def act(g, kind):
    """(act(g), act'(g)) in float64; kind: 0 g sigmoid(g), 1 g Phi(g), 2 max(g, 0)."""
    if kind == 0:
        s = 1 / (1 + np.exp(-g))
        return g * s, s + g * s * (1 - s)
    if kind == 1:
        p = np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in g.ravel()]).reshape(g.shape)
        return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return np.maximum(g, 0), (g > 0).astype(float)

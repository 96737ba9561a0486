"""Plain references of layer norm, the linear layer and the AdamW step (NumPy): 64 bits for the first two, and for
AdamW float32 with every operation rounded, which the step's results equal bit for bit."""
import numpy as np

import narrow_ref as ref

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # half a step, relative
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}                # half of the least float16


def layer_norm(x, w, b, eps):
    """(y, mean, rstd, xh) in float64."""
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    xh = (x - mean) * rstd
    return xh * w + b, mean, rstd, xh


def layer_norm_grad(dy, xh, rstd, w, add=0.0):
    a = dy * w
    dx = rstd * (a - a.mean(1, keepdims=True) - xh * (a * xh).mean(1, keepdims=True)) + add
    return dx, (dy * xh).sum(0), dy.sum(0)


def act(z, kind):
    """(act(z), act'(z)); kind None: z and 1."""
    return (z, np.ones_like(z)) if kind is None else ref.act(z, kind)


# ---- AdamW, float32 operations ----------------------------------------------

F = np.float32


def stirred(x):
    """32 bits (in uint64) stirred."""
    m = np.uint64(0xFFFFFFFF)
    x = np.asarray(x, dtype=np.uint64)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & m
    x = ((x ^ (x >> np.uint64(13))) * np.uint64(0x6A09E667)) & m
    return x ^ (x >> np.uint64(16))


def key(step, seed):
    k = np.uint64(0)
    for word in (step & 0xFFFFFFFF, step >> 32, seed & 0xFFFFFFFF, seed >> 32):
        k = stirred(k ^ np.uint64(word))
    return k


def uniform(places, step, seed):
    """The numbers for m and for r at these places of the states."""
    at = np.asarray(places, dtype=np.uint64)
    m = np.uint64(0xFFFFFFFF)
    k = key(step, seed) ^ ((at >> np.uint64(32)) * np.uint64(0x6A09E667) & m)
    h = stirred(((at & m) * np.uint64(0x9E3779B9) + k) & m)
    return ((h & np.uint64(0xFFFF)).astype(F) + F(0.5)) * F(2.0 ** -16), \
        ((h >> np.uint64(16)).astype(F) + F(0.5)) * F(2.0 ** -16)


def group_scales(x, f):
    """Scale exponents of groups of 32 of float32 values."""
    top = ref.code_values(f)[-1]
    a = np.abs(x.reshape(-1, 32)).astype(np.float64)
    a = np.where(np.isfinite(a), a, 0).max(1)
    k = np.full(len(a), -110)
    some = a > 0
    k[some] = np.maximum(-110, np.ceil(np.log2(a[some] / top)).astype(int) - 1)
    while True:
        over = np.ldexp(a, -k) > top
        if not over.any():
            return k
        k = k + over


def _codes(q, f):
    """Codes of scaled values that are codes' values."""
    v = ref.code_values(f)
    a = np.abs(q).astype(np.float64)
    i = np.searchsorted(v, np.where(np.isfinite(a), a, 0))
    full = 2 ** sum(f) - 1
    i = np.where(np.isfinite(a), i, full if f == (4, 3) else np.where(np.isnan(a), full, len(v)))
    return i, np.signbit(q)


def encode(x, u, f, square=None):
    """(codes, scale exponents, scaled values) of float32 x at random; square: x are the roots of these."""
    v = ref.code_values(f).astype(F)
    k = group_scales(x, f)
    s = np.ldexp(F(1), -k).astype(F).repeat(32)
    n = np.abs(x) * s
    fin = np.isfinite(n)
    i = np.searchsorted(v, np.where(fin, n, 0), side="right") - 1
    lo, hi = v[i], v[np.minimum(i + 1, len(v) - 1)]
    step = np.where(i + 1 < len(v), hi - lo, F(1))
    hi = lo + step
    with np.errstate(invalid="ignore", over="ignore"):
        if square is None:
            up = n / step - lo / step > u       # exact: both are multiples of a power of two
        else:
            up = square * s * s - lo * lo > u * (hi * hi - lo * lo)
    q = np.where(up, hi, lo)
    if square is not None:
        q = np.where((n > 0) & (q == 0), v[1], q)
    q = np.where(fin, q, n)
    codes, _ = _codes(q, f)
    return codes + (np.signbit(x).astype(np.int64) << sum(f)), k, np.copysign(q, x)


def decode(codes, scales, f):
    """float32 values of codes and scale bytes."""
    s = np.where(scales == 0, 2.0 ** -127, np.ldexp(1.0, scales.astype(int) - 127))
    return (ref.decode(codes, f).astype(F) * s.astype(F).repeat(32)).astype(F)


def adamw(p, g, m, v, step, lr, betas, eps, decay, scale=1.0):
    """(p, m, v, sqrt(v)) of float32 values."""
    b1, b2 = betas
    with np.errstate(all="ignore"):
        d = g * F(scale)
        m = m * F(b1) + d * F(1 - b1)
        v = v * F(b2) + d * d * F(1 - b2)
        r = np.sqrt(v)
        c1, c2 = (-np.expm1(step * np.log(b)) if b > 0 else 1.0 for b in (b1, b2))
        p = p * F(1 - lr * decay) - m / (r * F(1 / np.sqrt(c2)) + F(eps)) * F(lr / c1)
    return p, m, v, r

"""The operators around a gated feed-forward block in a training step, as measurable cases.

- Layer norm in front of the block: one pass ("norm"), and a training step's two ("norm_train": y; dx
  with the residual path's gradient added, and the gradients of weight and bias).
- The block's last projection, a matrix product with bias, activation and residual in its epilogue
  ("linear"), and a training step's passes ("linear_train": y; dx, dw and db).
- AdamW over all of a block's tensors at once ("adamw"): states in float32, or in 8 bits as blocks of
  32 values of one tensor with a power-of-two scale, m as it is and v by its square root.

An 8-bit state is rounded at random, so that it moves by less than a code's step on average: m to the
code above with the probability that keeps its mean, sqrt(v) with the one that keeps the mean of v (a
root that is not zero keeps the least code at least). The random numbers are a counter's: 32 bits
from the value's place, the step and a seed, the lower half for m, the upper half for v.
"""
import math

import torch

own = False  # True: the library's kernels, False: the plain form

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FMTS = {"e4m3": (4, 3), "e5m2": (5, 2)}
EPS = 1e-5                                     # of layer norm
LR, B1, B2, EPSILON, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01
SEED = 12345                                   # of the states' rounding
MAX_FLOPS = 1.2e12    # of a drawn product: the largest listed step's
MAX_VALUES = 1 << 26  # of a drawn norm
MAX_STATE = 1 << 27   # of a drawn optimiser's step


def _norm(name, kind, rows, cols, dtype, wtype, gap=0, add=False):
    """gap: values between the rows of x and dy (a part of a wider tensor)."""
    return _named(name, kind=kind, rows=rows, cols=cols, dtype=dtype, wtype=wtype, gap=gap, add=add)


def _linear(name, kind, T, K, N, dtype, act, bias=True, residual=False):
    return _named(name, kind=kind, T=T, K=K, N=N, dtype=dtype, act=act, bias=bias, residual=residual)


def _adamw(name, sizes, grad, states, copy="none"):
    """sizes: the tensors' numbers of values; copy: the type of a 16-bit copy of the weights."""
    return _named(name, kind="adamw", sizes=",".join(map(str, sizes)), grad=grad, states=states,
                  copy=copy)


def _named(name, **c):
    if name:
        c["name"] = name
    return c


def listed():
    block = [11264 * 4096] * 3 + [4096] * 3
    return [
        # serving: one token's norm, nothing but latency
        _norm("norm_token", "norm", 1, 4096, "bf16", "bf16"),
        # the norm of a long batch in training, the residual path's gradient joined
        _norm("norm_step", "norm_train", 16384, 4096, "bf16", "f32", add=True),
        # float32 activations of odd width, parts of a wider tensor
        _norm("norm_ragged_f32", "norm_train", 4097, 2731, "f32", "f32", gap=5),
        # serving: one token through the last projection, the weights read once
        _linear("linear_token", "linear", 1, 11264, 4096, "bf16", "none", residual=True),
        # a short ragged prompt with an activation
        _linear("linear_ragged", "linear", 333, 2730, 1000, "f16", "gelu"),
        # a long prompt through the last projection
        _linear("linear_prompt", "linear", 8192, 11264, 4096, "bf16", "none", residual=True),
        # a training step of a small layer on a short ragged batch: no size is a multiple of 8
        _linear("linear_train_ragged", "linear_train", 77, 1022, 2731, "f16", "silu"),
        # a training step of a large layer with an activation and a residual
        _linear("linear_train_step", "linear_train", 4096, 4096, 11264, "bf16", "gelu", residual=True),
        # a small block's step: three weights of 512 x 1408, norm and bias; latency counts
        _adamw("adamw_small", [512 * 1408] * 3 + [512] * 3, "f32", "f32"),
        # forty tensors of odd sizes in one call
        _adamw("adamw_many", [1 + 977 * (i * i % 41) for i in range(40)], "f16", "e5m2"),
        # a large block, bfloat16 gradients, and the copy that the next products read
        _adamw("adamw_block", block, "bf16", "f32", "bf16"),
        # the same with 8-bit states
        _adamw("adamw_block_8bit", block, "bf16", "e4m3", "bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: mostly a multiple of 64 or 8, sometimes any whole number."""
    n, m = _log(rng, lo, hi), rng.choice([64, 64, 8, 1])
    return max(lo, n // m * m)


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "norm_train", "linear", "linear", "linear_train",
                       "linear_train", "adamw", "adamw"])
    if kind in ("norm", "norm_train"):
        cols, dtype = _size(rng, 33, 16384), rng.choice(list(TYPES))
        return _norm(None, kind, _log(rng, 1, MAX_VALUES // cols), cols, dtype,
                     rng.choice([dtype, "f32"]), rng.choice([0, 0, 8, 5]), rng.random() < 0.5)
    if kind == "adamw":
        sizes, left = [], MAX_STATE
        for _ in range(_log(rng, 1, 64)):
            sizes.append(_log(rng, 1, max(1, left // 2)))
            left -= sizes[-1]
        return _adamw(None, sizes, rng.choice(list(TYPES)), rng.choice(["f32", "e4m3", "e5m2"]),
                      rng.choice(["none", "bf16", "f16"]))
    while True:
        c = _linear(None, kind, _log(rng, 1, 8192), _size(rng, 256, 16384), _size(rng, 256, 16384),
                    rng.choice(["bf16", "bf16", "f16"]), rng.choice(["none", "none", "silu", "gelu", "relu"]),
                    rng.random() < 0.5, rng.random() < 0.5)
        if work(c)["flops"] <= MAX_FLOPS:
            return c


# ---- inputs -----------------------------------------------------------------


def _activations(g, rows, cols, dtype, gap=0):
    """Rows of a layer's activations: normal values about a mean of their own, one column in 64 ten
    times as large, the rows' sizes spread over a factor of 4."""
    x = torch.randn((rows, cols + gap), generator=g, device=DEV)
    out = torch.rand((1, cols + gap), generator=g, device=DEV) < 1 / 64
    x = x * torch.where(out, 10.0, 1.0) + torch.randn((rows, 1), generator=g, device=DEV) / 4
    x = x * torch.exp2(torch.rand((rows, 1), generator=g, device=DEV) * 2 - 1)
    return x.to(TYPES[dtype])[:, :cols]


def _places(sizes):
    """Where each tensor begins in flat buffers, and their length: at multiples of 32."""
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += -(-n // 32) * 32
    return at, total


def _quantised(x, fmt):
    """Codes (uint8) and scales (uint8) of non-random blocks of 32 of float32 values: what a run of
    steps has left in the states."""
    top = 8 if fmt == "e4m3" else 15
    v = x.reshape(-1, 32)
    m, e = torch.frexp(v.abs().amax(1))
    k = (e - 1 - top + (2 * m > 1.75).int()).clamp(min=-110)
    k = torch.where(m > 0, k, torch.full_like(k, -110))
    n = (v * _pow2(-k)[:, None]).to(_type8(fmt))
    return n.view(torch.uint8).reshape(-1), (k + 127).to(torch.uint8)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": c}
    if c["kind"] in ("norm", "norm_train"):
        R, C = c["rows"], c["cols"]
        s["x"] = _activations(g, R, C, c["dtype"], c["gap"])
        s["w"] = (1 + torch.randn(C, generator=g, device=DEV) / 8).to(TYPES[c["wtype"]])
        s["b"] = (torch.randn(C, generator=g, device=DEV) / 8).to(TYPES[c["wtype"]])
        if c["kind"] == "norm_train":
            s["dy"] = _activations(g, R, C, c["dtype"], c["gap"]) / 64
            s["add"] = _activations(g, R, C, c["dtype"]) / 64 if c["add"] else None
        return s
    if c["kind"] in ("linear", "linear_train"):
        T, K, N, t = c["T"], c["K"], c["N"], TYPES[c["dtype"]]
        s["x"] = _activations(g, T, K, c["dtype"])
        s["w"] = (torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K)).to(t)
        s["b"] = (torch.randn(N, generator=g, device=DEV) / 8).to(t) if c["bias"] else None
        s["r"] = _activations(g, T, N, c["dtype"]) if c["residual"] else None
        if c["kind"] == "linear_train":
            s["dy"] = _activations(g, T, N, c["dtype"]) / 64
        return s
    sizes = [int(n) for n in c["sizes"].split(",")]
    at, total = _places(sizes)
    there = torch.zeros(total, device=DEV)
    for a, n in zip(at, sizes):
        there[a:a + n] = 1

    def flat(scale, spread):
        v = torch.randn(total, generator=g, device=DEV) * scale
        return v * torch.exp2(torch.rand(total, generator=g, device=DEV) * spread) * there

    s["p"] = flat(1 / 64, 0)
    s["g"] = flat(1e-3, 3).to(TYPES[c["grad"]])
    m, v = flat(2e-4, 3), flat(2e-3, 3).square()
    s["m"], s["v"] = (m, v) if c["states"] == "f32" else (
        _quantised(m, c["states"]), _quantised(v.sqrt(), c["states"]))
    s["copy"] = s["p"].to(TYPES[c["copy"]]) if c["copy"] != "none" else None
    s["step"] = 1000
    for name in ("p", "g", "copy"):
        if s[name] is not None:
            s[name + "s"] = [s[name][a:a + n] for a, n in zip(at, sizes)]
    return s


# ---- one pass ---------------------------------------------------------------


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2007_06563_amd import hobflops as hf
    c = s["case"]
    if c["kind"] == "norm":
        return hf.layer_norm(s["x"], s["w"], s["b"], EPS)
    if c["kind"] == "norm_train":
        y, saved = hf.layer_norm(s["x"], s["w"], s["b"], EPS, save=True)
        dx, dw, db = hf.layer_norm_backward(s["dy"], s["x"], saved, s["w"], add=s["add"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if c["kind"] in ("linear", "linear_train"):
        act = {"none": None, "silu": hf.GATE_SILU, "gelu": hf.GATE_GELU, "relu": hf.GATE_RELU}[c["act"]]
        if c["kind"] == "linear":
            return hf.linear(s["x"], s["w"], s["b"], act, residual=s["r"])
        y, z = hf.linear(s["x"], s["w"], s["b"], act, residual=s["r"], save=True)
        dx, dw, db = hf.linear_backward(s["dy"], s["x"], s["w"], z, act, db=c["bias"])
        out = {"y": y, "dx": dx, "dw": dw}
        return {**out, "db": db} if c["bias"] else out
    f = None if c["states"] == "f32" else FMTS[c["states"]]
    s["step"] += 1
    hf.adamw(s["ps"], s["gs"], hf.AdamWState(s["m"], s["v"], f), s["step"], lr=LR, betas=(B1, B2),
             eps=EPSILON, weight_decay=DECAY, copies=s.get("copys"), seed=SEED)
    out = {"p": s["p"], "copy": s["copy"]} if s["copy"] is not None else {"p": s["p"]}
    for name in ("m", "v"):
        t = s[name]
        if f is not None:
            n = t[0].numel()
            t = hf.block_unpack(t[0].view(1, n), t[1].view(1, n // 32), n, f, dtype=torch.bfloat16)[0]
        out[name] = t
    return out


def _pow2(e):
    """2^e in float32 for whole e in [-126, 127], exactly."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _type8(fmt):
    return torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2


def _act(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return torch.where(z > 0, z, torch.zeros_like(z)) if act == "relu" else z


def _act_grad(z, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return (z > 0).float()


def _mixed(x):
    """32 bits (in int64) stirred."""
    x = (x ^ (x >> 15)) * 0xBB67AE85 & 0xFFFFFFFF
    x = (x ^ (x >> 13)) * 0x6A09E667 & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(step, seed):
    k = 0
    for word in (step & 0xFFFFFFFF, step >> 32, seed & 0xFFFFFFFF, seed >> 32):
        k = _mixed(k ^ word)
    return k


def _halves(n, step):
    """Two uniform numbers of (0, 1) a value, multiples of 2^-17."""
    h = _mixed(torch.arange(n, device=DEV) * 0x9E3779B9 + _key(step, SEED) & 0xFFFFFFFF)
    return ((h & 0xFFFF).float() + 0.5) / 65536, ((h >> 16).float() + 0.5) / 65536


def _decoded(blocks, fmt):
    codes, scales = blocks
    v = codes.view(_type8(fmt)).float().reshape(-1, 32)
    return (v * _pow2(scales.int() - 127)[:, None]).reshape(-1)


def _encoded(x, u, fmt, root_of=None):
    """Stores nothing: (codes, scales, values) of x (or, where it is given, of the roots x of root_of,
    rounded up with the probability that keeps the mean of their squares)."""
    wE, wF = FMTS[fmt]
    top, low = (8, -6) if fmt == "e4m3" else (15, -14)
    v = x.reshape(-1, 32)
    m, e = torch.frexp(v.abs().amax(1))
    k = torch.where(m > 0, e - 1 - top + (2 * m > 1.75).int(), torch.full_like(e, -110)).clamp(min=-110)
    s = _pow2(-k)[:, None]
    n = (v * s).abs()
    step = _pow2((torch.frexp(n)[1] - 1).clamp(min=low) - wF)
    i = torch.floor(n / step)
    u = u.reshape(-1, 32)
    if root_of is None:
        q = (i + (n / step - i > u).float()) * step * torch.sign(v)
    else:
        square = root_of.reshape(-1, 32) * s * s
        a, b = i * step, i * step + step
        q = torch.where(square - a * a > u * (b * b - a * a), b, a)
        q = torch.where((n > 0) & (q == 0), _pow2(torch.full_like(k, low - wF))[:, None], q)
    codes = q.to(_type8(fmt)).view(torch.uint8)
    return codes.reshape(-1), (k + 127).to(torch.uint8), (q * _pow2(k)[:, None]).reshape(-1)


def _run_plain(s):
    c = s["case"]
    if c["kind"] in ("norm", "norm_train"):
        t, x, w = TYPES[c["dtype"]], s["x"].float(), s["w"].float()
        d = x - x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt(d.square().mean(1, keepdim=True) + EPS)
        xh = d * rstd
        y = (xh * w + s["b"].float()).to(t)
        if c["kind"] == "norm":
            return y
        dy = s["dy"].float()
        a = dy * w
        dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
        if s["add"] is not None:
            dx = dx + s["add"].float()
        return {"y": y, "dx": dx.to(t), "dw": (dy * xh).sum(0).to(s["w"].dtype),
                "db": dy.sum(0).to(s["w"].dtype)}
    if c["kind"] in ("linear", "linear_train"):
        t, x, w = TYPES[c["dtype"]], s["x"].float(), s["w"].float()
        z = x @ w.T
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z, c["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        if c["kind"] == "linear":
            return y.to(t)
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _act_grad(z, c["act"])
        out = {"y": y.to(t), "dx": (dz @ w).to(t), "dw": (dz.T @ x).to(t)}
        return {**out, "db": dz.sum(0).to(t)} if c["bias"] else out
    s["step"] += 1
    f, t = c["states"], s["step"]
    g = s["g"].float()
    m, r = (s["m"], s["v"]) if f == "f32" else (_decoded(s["m"], f), _decoded(s["v"], f))
    v = r if f == "f32" else r * r
    m = m * B1 + g * (1 - B1)
    v = v * B2 + g * g * (1 - B2)
    root = torch.sqrt(v)
    step = m / (root * (1 / math.sqrt(1 - B2 ** t)) + EPSILON) * (LR / (1 - B1 ** t))
    s["p"].copy_(s["p"] * (1 - LR * DECAY) - step)
    out = {"p": s["p"]}
    if s["copy"] is not None:
        out["copy"] = s["copy"].copy_(s["p"])
    if f == "f32":
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
        return out
    um, uv = _halves(m.numel(), t)
    for name, x, u, square in (("m", m, um, None), ("v", root, uv, v)):
        codes, scales, values = _encoded(x, u, f, square)
        s[name][0].copy_(codes)
        s[name][1].copy_(scales)
        out[name] = values.to(torch.bfloat16)
    return out


# ---- what a pass cannot do without ------------------------------------------


def _bytes(t):
    return 4 if t == "f32" else 2


def work(case):
    c = case
    if c["kind"] in ("norm", "norm_train"):
        n, e, w = c["rows"] * c["cols"], _bytes(c["dtype"]), c["cols"] * _bytes(c["wtype"])
        if c["kind"] == "norm":
            return {"bytes": 2 * e * n + 2 * w, "flops": 0.0}
        return {"bytes": (5 if c["add"] else 4) * e * n + 4 * w, "flops": 0.0}
    if c["kind"] in ("linear", "linear_train"):
        T, K, N = c["T"], c["K"], c["N"]
        more = (N if c["bias"] else 0) + (T * N if c["residual"] else 0)
        if c["kind"] == "linear":
            return {"bytes": 2 * (T * K + N * K + T * N + more), "flops": 2.0 * T * K * N}
        more += N if c["bias"] else 0
        return {"bytes": 2 * (2 * T * K + 2 * N * K + 2 * T * N + more), "flops": 6.0 * T * K * N}
    n = sum(int(n) for n in c["sizes"].split(","))
    more = 8 + _bytes(c["grad"]) + (2 if c["copy"] != "none" else 0)
    # 8-bit states: codes and scales read and written, and the values that they stand for
    return {"bytes": n * (more + (16 if c["states"] == "f32" else 8 + 4 / 32)), "flops": 0.0}


# ---- the same results from the definitions, in 64 bits ----------------------


def _gate64(z, act):
    """The activation and its derivative."""
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if act == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return (z.clamp(min=0), (z > 0).double()) if act == "relu" else (z, torch.ones_like(z))


def _norm64(c, s):
    x, w = s["x"].double(), s["w"].double()
    C = c["cols"]
    mean = x.sum(1, keepdim=True) / C
    var = torch.matmul((x - mean)[:, None, :], (x - mean)[:, :, None])[:, :, 0] / C
    deviation = torch.sqrt(var + EPS)
    xh = (x - mean) / deviation
    y = torch.addcmul(s["b"].double(), xh, w)
    if c["kind"] == "norm":
        return y
    dy = s["dy"].double()
    # the projections of dy w on the ones and on xh go
    a = dy * w
    a = a - a.sum(1, keepdim=True) / C - xh * ((a * xh).sum(1, keepdim=True) / C)
    dx = a / deviation
    if s["add"] is not None:
        dx += s["add"].double()
    return {"y": y, "dx": dx, "dw": torch.linalg.vecdot(dy, xh, dim=0), "db": torch.sum(dy, 0)}


def _state64(x, fmt, u, square):
    """What the codes of x stand for; square: x are roots, whose squares keep their mean."""
    wE, wF = FMTS[fmt]
    bias, values = 2 ** (wE - 1) - 1, []
    for code in range(2 ** (wE + wF)):
        e, f = code >> wF, code & (2 ** wF - 1)
        values.append(math.ldexp(f, 1 - bias - wF) if e == 0 else math.ldexp(2 ** wF + f, e - bias - wF))
    values = torch.tensor(values[:-1] if fmt == "e4m3" else values[:-(2 ** wF)], dtype=torch.float64,
                          device=x.device)
    top = values[-1]
    v = x.reshape(-1, 32)
    a = v.abs().amax(1, keepdim=True)
    k = torch.floor(torch.log2(a.clamp(min=1e-300) / top)) - 1
    for _ in range(2):
        k = torch.where(a * torch.exp2(-k) > top, k + 1, k)
    scale = torch.exp2(k.clamp(min=-110))
    n = v.abs() / scale
    i = torch.searchsorted(values, n.contiguous(), right=True) - 1   # values[i] <= n
    lo, hi = values[i], values[(i + 1).clamp(max=len(values) - 1)]
    if square:
        up = n * n - lo * lo > u.reshape(-1, 32) * (hi * hi - lo * lo)
    else:
        up = n - lo > u.reshape(-1, 32) * (hi - lo)
    q = torch.where(up, hi, lo)
    if square:
        q = torch.where((n > 0) & (q == 0), values[1], q)
    return (torch.copysign(q, v) * scale).reshape(-1)


def _uniform64(n, step, first):
    """The counter's numbers of the places first .. first + n - 1."""
    def stir(h):
        for shift, factor in ((15, 0xBB67AE85), (13, 0x6A09E667)):
            h = torch.bitwise_and((h ^ torch.bitwise_right_shift(h, shift)) * factor, 2 ** 32 - 1)
        return h ^ torch.bitwise_right_shift(h, 16)
    key = torch.zeros((), dtype=torch.int64, device=DEV)
    for word in (step % 2 ** 32, step // 2 ** 32, SEED % 2 ** 32, SEED // 2 ** 32):
        key = stir(key ^ word)
    h = stir(((torch.arange(n, device=DEV) + first) * 0x9E3779B9 + key) % 2 ** 32)
    return [(part.double() + 0.5) * 2.0 ** -16 for part in (h % 65536, h // 65536)]


def _adamw64(c, s):
    f, t = c["states"], s["step"] + 1
    p, g = s["p"].double(), s["g"].double()
    if f == "f32":
        m, v = s["m"].double(), s["v"].double()
    else:
        m, r = ((codes.view(_type8(f)).double().reshape(-1, 32) *
                 torch.exp2(scales.double() - 127)[:, None]).reshape(-1) for codes, scales in (s["m"], s["v"]))
        v = r.square()
    m = torch.lerp(g, m, B1)
    v = torch.lerp(g.square(), v, B2)
    p = p - LR * DECAY * p
    p = p - LR * (m / (1 - B1 ** t)) / (torch.sqrt(v / (1 - B2 ** t)) + EPSILON)
    out = {"p": p, "copy": p} if s["copy"] is not None else {"p": p}
    if f == "f32":
        return {**out, "m": m, "v": v}
    root, part = torch.sqrt(v), 1 << 25     # in parts, to hold the temporaries down
    for a in range(0, len(m), part):
        e = min(len(m), a + part)
        um, uv = _uniform64(e - a, t, a)
        m[a:e] = _state64(m[a:e], f, um, False)
        root[a:e] = _state64(root[a:e], f, uv, True)
    return {**out, "m": m, "v": root}


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("norm", "norm_train"):
        return _norm64(c, s)
    if c["kind"] == "adamw":
        return _adamw64(c, s)
    x, w = s["x"].double(), s["w"].double()
    z = torch.matmul(x, w.t())
    if s["b"] is not None:
        z += s["b"].double()
    a, d = _gate64(z, c["act"])
    y = a + s["r"].double() if s["r"] is not None else a
    if c["kind"] == "linear":
        return y
    dz = s["dy"].double() * d
    out = {"y": y, "dx": torch.matmul(dz, w), "dw": torch.matmul(dz.t(), x)}
    return {**out, "db": torch.sum(dz, 0)} if c["bias"] else out

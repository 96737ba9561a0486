"""The operators of a gated feed-forward block on group-scaled narrow floats, as measurable cases.

A network's block is trained and then served:

- its activations are kept for the backward pass as 8-bit floats with one power-of-two scale a
  group of 32 ("ckpt": what a layer hands over, packed and read back);
- h = act(x Wg^T) * (x Wu^T) ("forward"), and a training step that keeps x and both projections
  in 8 bits and computes the gradients of x and of both weights from them ("train");
- its weights are served as 4-bit floats with one scale a group of 32, 64 or 128, for a few
  tokens at a time ("w4": one projection, "w4_gated": both, the activation and the product).

The 8-bit codes are the formats (4, 3) and (5, 2), the 4-bit ones (2, 1): sign, exponent,
fraction, subnormal values where the exponent is 0. (4, 3) gives one code a sign to NaN and has
no infinity, (5, 2) keeps both in its highest exponent, (2, 1) has neither.
"""
import math

import torch

own = False  # True: the library's kernels, False: the plain form

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FMTS = {"e4m3": (4, 3), "e5m2": (5, 2)}
MAX_FLOPS = 2.2e12   # of a drawn pass: the largest listed step's
MAX_VALUES = 1 << 26  # of a drawn checkpoint


def _ckpt(name, rows, cols, dtype, fmt, gap=0):
    """gap: values between the rows (a part of a wider tensor)."""
    return _named(name, kind="ckpt", rows=rows, cols=cols, dtype=dtype, fmt=fmt, gap=gap)


def _gated(name, kind, T, D, F, dtype, act, fmt="none"):
    return _named(name, kind=kind, T=T, D=D, F=F, dtype=dtype, act=act, fmt=fmt)


def _w4(name, kind, T, K, N, dtype, group, scale, act="none"):
    return _named(name, kind=kind, T=T, K=K, N=N, dtype=dtype, group=group, scale=scale, act=act)


def _named(name, **c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token's activations: the smallest call, nothing but latency
        _ckpt("ckpt_token", 1, 4096, "bf16", "e4m3"),
        # a layer's activations for a long batch
        _ckpt("ckpt_layer", 16384, 4096, "bf16", "e4m3"),
        # float32 activations of odd width, a part of a wider tensor, in the format of more range
        _ckpt("ckpt_ragged_f32", 4097, 2731, "f32", "e5m2", gap=5),
        # a token through the block: both weights are read once
        _gated("forward_token", "forward", 1, 4096, 11264, "bf16", "silu"),
        # a short ragged prompt through a small block
        _gated("forward_ragged", "forward", 333, 1000, 2730, "f16", "gelu"),
        # a long prompt: the largest matrix products of inference
        _gated("forward_prompt", "forward", 8192, 4096, 11264, "bf16", "silu"),
        # a training step of a small block on a short ragged batch: no size is a multiple of 8
        _gated("train_ragged", "train", 77, 1022, 2731, "f16", "gelu", "e5m2"),
        # a training step of a large one
        _gated("train_step", "train", 4096, 4096, 11264, "bf16", "silu", "e4m3"),
        # serving: one token through a square projection
        _w4("w4_token", "w4", 1, 4096, 4096, "bf16", 128, "bf16"),
        # sixteen requests at once through the block's last projection
        _w4("w4_batch", "w4", 16, 11264, 4096, "f16", 32, "pow2"),
        # a few tokens through an output layer of odd width, its last group not whole
        _w4("w4_head", "w4", 5, 4104, 50257, "bf16", 64, "f32"),
        # one token through both projections, the activation and the product
        _w4("w4_gated_token", "w4_gated", 1, 4096, 11264, "bf16", 32, "pow2", "silu"),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """A width: mostly a multiple of 64 or 8, sometimes any whole number."""
    n, m = _log(rng, lo, hi), rng.choice([64, 64, 8, 1])
    return max(lo, n // m * m)


def draw(rng):
    kind = rng.choice(["ckpt", "forward", "forward", "train", "train", "w4", "w4", "w4_gated"])
    if kind == "ckpt":
        cols = _size(rng, 33, 16384)
        return _ckpt(None, _log(rng, 1, MAX_VALUES // cols), cols, rng.choice(list(TYPES)),
                     rng.choice(list(FMTS)), rng.choice([0, 0, 8, 5]))
    if kind in ("forward", "train"):
        act, dtype = rng.choice(["silu", "silu", "gelu", "relu"]), rng.choice(["bf16", "bf16", "f16"])
        while True:
            c = _gated(None, kind, _log(rng, 1, 8192), _size(rng, 256, 8192),
                       _size(rng, 512, 16384), dtype, act,
                       rng.choice(list(FMTS)) if kind == "train" else "none")
            if work(c)["flops"] <= MAX_FLOPS:
                return c
    return _w4(None, kind, _log(rng, 1, 64), max(256, _size(rng, 256, 16384) // 8 * 8),
               _size(rng, 256, 32768), rng.choice(["bf16", "f16"]), rng.choice([32, 64, 128]),
               rng.choice(["pow2", "bf16", "f32"]),
               rng.choice(["silu", "gelu", "relu"]) if kind == "w4_gated" else "none")


# ---- inputs -----------------------------------------------------------------


def _activations(g, rows, cols, dtype, gap=0):
    """Rows of a layer's activations: normal values, one column in 64 ten times as large (the
    columns that stand out in a trained network), the rows' sizes spread over a factor of 4."""
    x = torch.randn((rows, cols + gap), generator=g, device=DEV)
    out = torch.rand((1, cols + gap), generator=g, device=DEV) < 1 / 64
    x = x * torch.where(out, 10.0, 1.0)
    x = x * torch.exp2(torch.rand((rows, 1), generator=g, device=DEV) * 2 - 1)
    return x.to(TYPES[dtype])[:, :cols]


def _weight(g, rows, cols, dtype):
    return (torch.randn((rows, cols), generator=g, device=DEV) / math.sqrt(cols)).to(TYPES[dtype])


def _weight4(g, rows, cols, group, scale):
    """4-bit codes [rows, cols / 2] (the even element in the low half of a byte) and scales
    [rows, groups] of a normal weight: a group's largest value takes the largest code, 6."""
    groups = -(-cols // group)
    codes = torch.randint(0, 256, (rows, -(-cols // 2)), generator=g, device=DEV,
                          dtype=torch.uint8)
    s = torch.rand((rows, groups), generator=g, device=DEV) + 0.5
    s = s / (6 * math.sqrt(cols)) * 3
    if scale == "pow2":
        return codes, (torch.floor(torch.log2(s)) + 127).to(torch.uint8)
    return codes, s.to(TYPES[scale])


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "ckpt":
        s["x"] = _activations(g, c["rows"], c["cols"], c["dtype"], c["gap"])
    elif c["kind"] in ("forward", "train"):
        s["x"] = _activations(g, c["T"], c["D"], c["dtype"])
        s["w_gate"] = _weight(g, c["F"], c["D"], c["dtype"])
        s["w_up"] = _weight(g, c["F"], c["D"], c["dtype"])
        if c["kind"] == "train":
            s["dh"] = _activations(g, c["T"], c["F"], c["dtype"]) / 64
    else:
        s["x"] = _activations(g, c["T"], c["K"], c["dtype"])
        s["w"] = _weight4(g, c["N"], c["K"], c["group"], c["scale"])
        if c["kind"] == "w4_gated":
            s["w_up"] = _weight4(g, c["N"], c["K"], c["group"], c["scale"])
    return s


# ---- one pass ---------------------------------------------------------------


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2007_06563_amd import hobflops as hf
    c = s["case"]
    act = {"none": None, "silu": hf.GATE_SILU, "gelu": hf.GATE_GELU, "relu": hf.GATE_RELU}[
        c.get("act", "none")]
    if c["kind"] == "ckpt":
        f = FMTS[c["fmt"]]
        codes, scales = hf.block_pack(s["x"], f)
        return hf.block_unpack(codes, scales, c["cols"], f, dtype=s["x"].dtype)
    if c["kind"] == "forward":
        return hf.gated_forward(s["x"], s["w_gate"], s["w_up"], act)
    if c["kind"] == "train":
        h, saved = hf.gated_forward(s["x"], s["w_gate"], s["w_up"], act, ckpt=FMTS[c["fmt"]])
        dx, dw_gate, dw_up = hf.gated_backward(s["dh"], saved, s["w_gate"], s["w_up"], act)
        return {"h": h, "dx": dx, "dw_gate": dw_gate, "dw_up": dw_up}
    if c["kind"] == "w4":
        return hf.w4_linear(s["x"], *s["w"], group=c["group"])
    return hf.w4_gated(s["x"], *s["w"], *s["w_up"], act, group=c["group"])


def _pow2(e):
    """2^e in float32 for whole e in [-126, 127], exactly."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _through_8_bits(x, fmt):
    """float32 values as the format's codes hold them, under a scale 2^k a group of 32 of a row:
    k the smallest (but at least -110) for which no finite value of the group rounds beyond the
    format's largest."""
    wE, wF = FMTS[fmt]
    bias = 2 ** (wE - 1) - 1
    top = 8 if fmt == "e4m3" else 15          # exponent of the largest value, 1.75 * 2^top
    rows, cols = x.shape
    v = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)
    a = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v)).amax(2, keepdim=True)
    m, e = torch.frexp(a)                     # a = m 2^e, m in [0.5, 1)
    over = 2 * m > 1.8125 if fmt == "e4m3" else 2 * m >= 1.875
    k = torch.where(a > 0, e - 1 - top + over.int(), torch.full_like(e, -110)).clamp(min=-110)
    n = v * _pow2(-k)
    step = _pow2((torch.frexp(n)[1] - 1).clamp(1 - bias, top + 1) - wF)
    q = torch.round(n / step) * step
    lost = torch.full_like(v, math.nan)
    q = torch.where(torch.isfinite(v), q, lost if fmt == "e4m3" else v) * _pow2(k)
    return q.reshape(rows, -1)[:, :cols]


def _act(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    if act == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    return torch.where(g > 0, g, torch.where(torch.isnan(g), g, torch.zeros_like(g)))


def _act_grad(g, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    return torch.where(g > 0, torch.ones_like(g), torch.where(torch.isnan(g), g, torch.zeros_like(g)))


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _decode4(codes, scales, cols, group):
    """The weights that 4-bit codes stand for, float32 [rows, cols]."""
    table = torch.tensor(_E2M1 + [-v for v in _E2M1], device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1)[:, :cols]
    s = _pow2(scales.int() - 127) if scales.dtype == torch.uint8 else scales.float()
    return table[both.long()] * s.repeat_interleave(group, 1)[:, :cols]


def _run_plain(s):
    c, t = s["case"], TYPES[s["case"]["dtype"]]
    x = s["x"].float()
    if c["kind"] == "ckpt":
        return _through_8_bits(x, c["fmt"]).to(t)
    if c["kind"] in ("forward", "train"):
        wg, wu = s["w_gate"].float(), s["w_up"].float()
        g, u = x @ wg.T, x @ wu.T
        h = (_act(g, c["act"]) * u).to(t)
        if c["kind"] == "forward":
            return h
        x, g, u = (_through_8_bits(v, c["fmt"]) for v in (x, g, u))
        dh = s["dh"].float()
        dg, du = dh * u * _act_grad(g, c["act"]), dh * _act(g, c["act"])
        return {"h": h, "dx": (dg @ wg + du @ wu).to(t), "dw_gate": (dg.T @ x).to(t),
                "dw_up": (du.T @ x).to(t)}
    y = x @ _decode4(*s["w"], c["K"], c["group"]).T
    if c["kind"] == "w4":
        return y.to(t)
    return (_act(y, c["act"]) * (x @ _decode4(*s["w_up"], c["K"], c["group"]).T)).to(t)


# ---- what a pass cannot do without ------------------------------------------


def work(case):
    c = case
    b = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "ckpt":
        n = c["rows"] * c["cols"]
        return {"bytes": 2 * b * n + n + c["rows"] * -(-c["cols"] // 32), "flops": 0.0}
    if c["kind"] in ("forward", "train"):
        T, D, F = c["T"], c["D"], c["F"]
        if c["kind"] == "forward":
            return {"bytes": b * (T * D + 2 * F * D + T * F), "flops": 4.0 * T * D * F}
        return {"bytes": b * (2 * T * D + 4 * F * D + 2 * T * F), "flops": 12.0 * T * D * F}
    T, K, N = c["T"], c["K"], c["N"]
    n = 2 if c["kind"] == "w4_gated" else 1
    scale = {"pow2": 1, "bf16": 2, "f32": 4}[c["scale"]]
    w = N * -(-K // 2) + N * -(-K // c["group"]) * scale
    return {"bytes": n * w + b * (T * K + T * N), "flops": 2.0 * n * T * K * N}


# ---- the same results from the definitions, in 64 bits ----------------------


def _code_values(fmt):
    """The finite non-negative values of a format's codes, ascending (the code is the index)."""
    wE, wF = FMTS[fmt]
    bias, values = 2 ** (wE - 1) - 1, []
    for code in range(2 ** (wE + wF)):
        e, f = code >> wF, code & (2 ** wF - 1)
        values.append(math.ldexp(f, 1 - bias - wF) if e == 0 else
                      math.ldexp(2 ** wF + f, e - bias - wF))
    return values[:-1] if fmt == "e4m3" else values[:-(2 ** wF)]


def _nearest(x, fmt):
    """float64 values as their group's codes hold them: every value goes to the nearest code under
    the group's scale, the even one of two."""
    values = _code_values(fmt)
    t = torch.tensor(values, dtype=torch.float64, device=x.device)
    mid = (t[1:] + t[:-1]) / 2
    # the first value beyond the largest: what rounds up to the step above it
    limit = (values[-1] + 2 * values[-1] - values[-2]) / 2
    rows, cols = x.shape
    out = torch.empty_like(x)
    for c0 in range(0, cols, 4096):           # columns in parts, to hold the temporaries down
        v = x[:, c0:c0 + 4096]
        w = v.shape[1]
        v = torch.nn.functional.pad(v, (0, -w % 32)).reshape(rows, -1, 32)
        a = torch.nan_to_num(v.abs(), nan=0.0, posinf=0.0).amax(2, keepdim=True)
        k = torch.floor(torch.log2(a.clamp(min=1e-300) / limit)) - 1
        for _ in range(3):
            n = a * torch.exp2(-k)
            k = torch.where((n > limit) | ((n == limit) & (fmt == "e5m2")), k + 1, k)
        scale = torch.exp2(k.clamp(min=-110))
        n = v.abs() / scale
        i = torch.bucketize(n, mid, right=False)   # mid[i - 1] < n <= mid[i]
        at = mid[i.clamp(max=len(mid) - 1)]
        i = torch.where((n == at) & (i < len(mid)) & (i % 2 == 1), i + 1, i)
        q = torch.copysign(t[i], v) * scale
        bad = v if fmt == "e5m2" else torch.full_like(v, math.nan)
        q = torch.where(torch.isfinite(v), q, bad)
        out[:, c0:c0 + 4096] = q.reshape(rows, -1)[:, :w]
    return out


def _normal_cdf(g):
    return torch.special.ndtr(g)


def _gate64(g, act):
    """The activation and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * torch.sigmoid(-g)
    if act == "gelu":
        p = _normal_cdf(g)
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g.clamp(min=0), (g > 0).double()


def _weights64(codes, scales, cols, group):
    """sign (-1)^s, exponent e, fraction f: f / 2 for e = 0, else (1 + f / 2) 2^(e - 1)."""
    q = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.int64, device=codes.device)
    q[:, 0::2], q[:, 1::2] = codes & 15, codes >> 4
    q = q[:, :cols]
    e, f = (q >> 1) & 3, (q & 1).double()
    v = torch.where(e == 0, f / 2, (1 + f / 2) * torch.exp2(e.double() - 1))
    v = torch.where(q >= 8, -v, v)
    s = torch.exp2(scales.double() - 127) if scales.dtype == torch.uint8 else scales.double()
    return v * s[:, torch.arange(cols, device=codes.device) // group]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    x = s["x"].double()
    if c["kind"] == "ckpt":
        return _nearest(x, c["fmt"])
    if c["kind"] in ("forward", "train"):
        wg, wu = s["w_gate"].double(), s["w_up"].double()
        g, u = torch.matmul(x, wg.t()), torch.matmul(x, wu.t())
        h = _gate64(g, c["act"])[0] * u
        if c["kind"] == "forward":
            return h
        x, g, u = _nearest(x, c["fmt"]), _nearest(g, c["fmt"]), _nearest(u, c["fmt"])
        a, d = _gate64(g, c["act"])
        dh = s["dh"].double()
        both = torch.cat([dh * u * d, dh * a], 1)             # [T, 2 F]
        dx = torch.matmul(both, torch.cat([wg, wu], 0))
        dw = torch.matmul(both.t(), x)
        return {"h": h, "dx": dx, "dw_gate": dw[:c["F"]], "dw_up": dw[c["F"]:]}
    y = torch.matmul(x, _weights64(*s["w"], c["K"], c["group"]).t())
    if c["kind"] == "w4":
        return y
    up = torch.matmul(x, _weights64(*s["w_up"], c["K"], c["group"]).t())
    return _gate64(y, c["act"])[0] * up

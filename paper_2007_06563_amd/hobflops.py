"""Python binding of libhobflops.so (ctypes).

Argument marshalling only: every step runs in the library's HIP kernels, on
torch's current stream; torch supplies device memory and streams. There is no
CPU fallback: a missing library or a host tensor raises.
Plane tensors are int32 (the bit patterns of PL32 words).
"""
import collections
import ctypes
import os
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhobflops.so")
_lib = None

SRC_F32, SRC_CODE_U32 = 0, 1
ACT_NONE, ACT_RELU = 0, 1
ROUND_NEAREST_EVEN, ROUND_TOWARD_ZERO, ORDER_KY_KX_C = 0, 1, 0
ALGO_AUTO, ALGO_FUSED, ALGO_SPLIT, ALGO_SPLIT_COMPACT = 0, 1, 2, 3
OFM_PLANES, OFM_F32, OFM_CODE = 0, 1, 2
TILE_112X64, TILE_56X64, TILE_32X64, TILE_32X32, TILE_16X32 = 1, 2, 3, 4, 5
SCALE_POW2, SCALE_BF16, SCALE_F32 = 0, 1, 2
GATE_SILU, GATE_GELU, GATE_RELU = 0, 1, 2
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_SCALES = {torch.uint8: SCALE_POW2, torch.bfloat16: SCALE_BF16, torch.float32: SCALE_F32}
_SCALE_TYPES = {v: k for k, v in _SCALES.items()}


class HobflopsError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"hobflops status {status}: {msg}")
        self.status = status


class Fmt(ctypes.Structure):
    _fields_ = [("wE", ctypes.c_int), ("wF", ctypes.c_int)]

    def __repr__(self):
        return f"Fmt({self.wE}, {self.wF})"


class ConvDesc(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int), ("H", ctypes.c_int), ("W", ctypes.c_int),
                ("C", ctypes.c_int), ("M", ctypes.c_int), ("KH", ctypes.c_int),
                ("KW", ctypes.c_int), ("stride", ctypes.c_int), ("pad", ctypes.c_int),
                ("in_fmt", Fmt), ("acc_fmt", Fmt), ("out_fmt", Fmt),
                ("act", ctypes.c_int), ("round", ctypes.c_int), ("order", ctypes.c_int),
                ("algo", ctypes.c_int), ("ofm_kind", ctypes.c_int)]


class PackJob(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("kind", ctypes.c_int), ("rows", ctypes.c_int64),
                ("len", ctypes.c_int64), ("planes", ctypes.c_void_p)]


class GatedDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int64), ("D", ctypes.c_int64), ("F", ctypes.c_int64),
                ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64), ("ldh", ctypes.c_int64),
                ("type", ctypes.c_int), ("act", ctypes.c_int), ("ckpt", Fmt),
                ("align", ctypes.c_int)]


# What gated_forward keeps for gated_backward: (codes, scales) of x, g and u.
GatedSaved = collections.namedtuple("GatedSaved", "x gate up fmt")


EXPORTS = ("hobflops_plane_words", "hobflops_pack", "hobflops_pack_batch", "hobflops_unpack",
           "hobflops_conv2d",
           "hobflops_conv2d_supported", "hobflops_conv2d_algo", "hobflops_conv2d_value_ops",
           "hobflops_conv2d_value_tile", "hobflops_conv2d_on_values",
           "hobflops_muladd", "hobflops_muladd_supported",
           "hobflops_netlist_ops", "hobflops_avgpool", "hobflops_avgpool_supported",
           "hobflops_avgpool_netlist_ops", "hobflops_block_pack", "hobflops_block_unpack",
           "hobflops_gated_workspace", "hobflops_gated_forward", "hobflops_gated_backward",
           "hobflops_w4_linear", "hobflops_w4_gated", "hobflops_wait_failures", "hobflops_set_wait_limit",
           "hobflops_get_wait_limit", "hobflops_status_string")


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2007_06563_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        L.hobflops_plane_words.argtypes = [i64, i64, Fmt, ctypes.POINTER(i64)]
        L.hobflops_pack.argtypes = [vp, ci, i64, i64, Fmt, vp, vp]
        L.hobflops_pack_batch.argtypes = [ctypes.POINTER(PackJob), ci, Fmt, vp]
        L.hobflops_unpack.argtypes = [vp, i64, i64, Fmt, ci, vp, vp]
        L.hobflops_conv2d.argtypes = [vp, vp, vp, ctypes.POINTER(ConvDesc), vp]
        L.hobflops_conv2d_supported.argtypes = [ctypes.POINTER(ConvDesc)]
        L.hobflops_conv2d_algo.argtypes = [ctypes.POINTER(ConvDesc)]
        L.hobflops_conv2d_value_ops.argtypes = [ctypes.POINTER(ConvDesc)]
        L.hobflops_conv2d_value_tile.argtypes = [ctypes.POINTER(ConvDesc)]
        L.hobflops_conv2d_on_values.argtypes = [vp, vp, vp, ctypes.POINTER(ConvDesc), ci, vp]
        L.hobflops_muladd.argtypes = [vp, vp, vp, vp, i64, Fmt, Fmt, ci, vp]
        L.hobflops_muladd_supported.argtypes = [Fmt, Fmt, ci]
        L.hobflops_netlist_ops.argtypes = [Fmt, Fmt, ci] + [ctypes.POINTER(ci)] * 4
        L.hobflops_avgpool.argtypes = [vp, vp, ci, ci, ci, ci, Fmt, Fmt, Fmt, ci, vp]
        L.hobflops_avgpool_supported.argtypes = [Fmt, Fmt, Fmt, ci]
        L.hobflops_avgpool_netlist_ops.argtypes = [Fmt, Fmt, Fmt, ci] + [ctypes.POINTER(ci)] * 2
        L.hobflops_block_pack.argtypes = [vp, ci, i64, i64, i64, Fmt, ci, ci, vp, vp, vp]
        L.hobflops_block_unpack.argtypes = [vp, vp, i64, i64, Fmt, ci, ci, vp, ci, i64, vp]
        L.hobflops_gated_workspace.argtypes = [ctypes.POINTER(GatedDesc), ci, ctypes.POINTER(i64)]
        L.hobflops_gated_forward.argtypes = [ctypes.POINTER(GatedDesc)] + [vp] * 9 + [i64, vp]
        L.hobflops_gated_backward.argtypes = [ctypes.POINTER(GatedDesc)] + [vp] * 13 + [i64, vp]
        L.hobflops_w4_linear.argtypes = [vp, ci, i64, i64, i64, i64, vp, vp, ci, ci, vp, i64, vp]
        L.hobflops_w4_gated.argtypes = [vp, ci, i64, i64, i64, i64, vp, vp, vp, vp, ci, ci, ci, vp,
                                        i64, vp]
        L.hobflops_wait_failures.argtypes = [ctypes.POINTER(ctypes.c_uint32), ci]
        L.hobflops_set_wait_limit.argtypes = [ctypes.c_uint32]
        L.hobflops_get_wait_limit.argtypes = []
        L.hobflops_status_string.argtypes = [ci]
        L.hobflops_status_string.restype = ctypes.c_char_p
        for name in EXPORTS[:-1]:
            getattr(L, name).restype = ci
        L.hobflops_get_wait_limit.restype = ctypes.c_uint32
        _lib = L
    return _lib


def fmt(f):
    return f if isinstance(f, Fmt) else Fmt(int(f[0]), int(f[1]))


def nb(f):
    f = fmt(f)
    return 3 + f.wE + f.wF


def _check(rc):
    if rc != 0:
        raise HobflopsError(rc, lib().hobflops_status_string(rc).decode())


def _ptr(t):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("hobflops operates on GPU tensors only")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _require(t, nbytes, name):
    """The library reads and writes through raw pointers: a tensor smaller than
    the call's extent is refused here, before any launch."""
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise ValueError(f"{name}: {have} bytes, the call needs {nbytes}")


def _call(device, function, *args):
    """function(*args, stream) on the device's current stream, with the device as the current one: a
    launch on the default stream goes to whichever device is current. (The raw handle:
    torch.cuda.current_stream would make an object of it, at 2 us a call.)"""
    stream = torch._C._cuda_getCurrentRawStream(device.index)
    if torch._C._cuda_getDevice() == device.index:
        rc = function(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = function(*args, stream)
    if rc:
        _check(rc)


def plane_words(rows, length, f):
    w = ctypes.c_int64()
    _check(lib().hobflops_plane_words(rows, length, fmt(f), ctypes.byref(w)))
    return w.value


def plane_shape(rows, length, f):
    return (rows, (length + 31) // 32, nb(f))


def pack(src, f, rows=None, length=None, out=None):
    """float32 values or int32 codes [rows, length] (any shape whose last axis
    is the packed one) -> int32 planes [rows, ceil(length/32), NB]."""
    f = fmt(f)
    if length is None:
        length = src.shape[-1]
    if rows is None:
        rows = src.numel() // max(length, 1)
    if src.numel() != rows * length:
        raise ValueError("rows * length does not match the source size")
    if src.dtype == torch.float32:
        kind = SRC_F32
    elif src.dtype in (torch.int32, torch.uint32):
        kind = SRC_CODE_U32
    else:
        raise TypeError("pack takes float32 values or int32 codes")
    if out is None:
        out = torch.empty(plane_shape(rows, length, f), dtype=torch.int32, device=src.device)
    _require(out, 4 * plane_words(rows, length, f), "pack out")
    _call(src.device, lib().hobflops_pack, _ptr(src), kind, rows, length, f, _ptr(out))
    return out


def pack_batch(items, f):
    """Several pack() calls of one format in one launch (per 8 tensors).
    items: sequence of (src, out) pairs with out None or a planes tensor, or
    bare src tensors; each src packed along its last axis, as pack() does.
    Returns the planes tensors in order. The launch goes to the current stream
    of the first source's device."""
    f = fmt(f)
    jobs, outs = [], []
    for it in items:
        src, out = it if isinstance(it, (tuple, list)) else (it, None)
        length = src.shape[-1] if src.dim() else 1
        rows = src.numel() // max(length, 1)
        if src.dtype == torch.float32:
            kind = SRC_F32
        elif src.dtype in (torch.int32, torch.uint32):
            kind = SRC_CODE_U32
        else:
            raise TypeError("pack takes float32 values or int32 codes")
        if out is None:
            out = torch.empty(plane_shape(rows, length, f), dtype=torch.int32, device=src.device)
        _require(out, 4 * plane_words(rows, length, f), "pack_batch out")
        jobs.append(PackJob(_ptr(src).value, kind, rows, length, _ptr(out).value))
        outs.append(out)
    if not jobs:
        return outs
    arr = (PackJob * len(jobs))(*jobs)
    first = items[0][0] if isinstance(items[0], (tuple, list)) else items[0]
    _call(first.device, lib().hobflops_pack_batch, arr, len(jobs), f)
    return outs


def unpack(planes, rows, length, f, kind="f32", out=None):
    """int32 planes -> float32 values (kind 'f32') or int32 codes ('code'), [rows, length]."""
    f = fmt(f)
    k = SRC_F32 if kind == "f32" else SRC_CODE_U32
    if out is None:
        out = torch.empty((rows, length), dtype=torch.float32 if k == SRC_F32 else torch.int32,
                          device=planes.device)
    _require(planes, 4 * plane_words(rows, length, f), "unpack planes")
    _require(out, 4 * rows * length, "unpack out")
    _call(planes.device, lib().hobflops_unpack, _ptr(planes), rows, length, f, k, _ptr(out))
    return out


def conv_desc(N, H, W, C, M, KH, KW, stride, pad, in_fmt, acc_fmt, out_fmt, act=ACT_NONE,
              algo=ALGO_AUTO, round=ROUND_NEAREST_EVEN, ofm_kind=OFM_PLANES):
    return ConvDesc(N, H, W, C, M, KH, KW, stride, pad, fmt(in_fmt), fmt(acc_fmt), fmt(out_fmt),
                    act, round, ORDER_KY_KX_C, algo, ofm_kind)


def conv_out_hw(d):
    return ((d.H + 2 * d.pad - d.KH) // d.stride + 1, (d.W + 2 * d.pad - d.KW) // d.stride + 1)


def _conv_out(ifm, w, d, out):
    """conv2d's output tensor (a new one for None), all three checked."""
    OH, OW = conv_out_hw(d)
    if out is None:
        if d.ofm_kind == OFM_PLANES:
            out = torch.empty(plane_shape(d.N * OH * OW, d.M, d.out_fmt), dtype=torch.int32,
                              device=ifm.device)
        else:
            out = torch.empty((d.N * OH * OW, d.M), device=ifm.device,
                              dtype=torch.float32 if d.ofm_kind == OFM_F32 else torch.int32)
    if OH > 0 and OW > 0 and d.N > 0 and d.C > 0 and d.M > 0:
        _require(ifm, 4 * plane_words(d.N * d.H * d.W, d.C, d.in_fmt), "conv2d ifm")
        _require(w, 4 * plane_words(d.KH * d.KW * d.C, d.M, d.in_fmt), "conv2d w")
        _require(out, 4 * (plane_words(d.N * OH * OW, d.M, d.out_fmt) if d.ofm_kind == OFM_PLANES
                           else d.N * OH * OW * d.M), "conv2d out")
    return out


def conv2d(ifm, w, d, out=None):
    """ifm planes [N*H*W, ceil(C/32), NB_in], w planes [KH*KW*C, ceil(M/32), NB_in]
    -> ofm planes [N*OH*OW, ceil(M/32), NB_out]; with d.ofm_kind OFM_F32 / OFM_CODE,
    float32 values / int32 codes [N*OH*OW, M]."""
    out = _conv_out(ifm, w, d, out)
    _call(ifm.device, lib().hobflops_conv2d, _ptr(ifm), _ptr(w), _ptr(out), ctypes.byref(d))
    return out


def conv2d_supported(d):
    return bool(lib().hobflops_conv2d_supported(ctypes.byref(d)))


def conv2d_algo(d):
    """The bitsliced kernel shape (ALGO_FUSED, ALGO_SPLIT or ALGO_SPLIT_COMPACT)
    of d: d.algo, or what AUTO picks on the current device unless it runs d on
    float32 values (conv2d_value_ops)."""
    rc = lib().hobflops_conv2d_algo(ctypes.byref(d))
    if rc < 0:
        _check(rc)
    return rc


def conv2d_value_ops(d):
    """Operations of one multiply-add where ALGO_AUTO runs d on float32 values, one
    per lane, instead of bitsliced; else 0."""
    rc = lib().hobflops_conv2d_value_ops(ctypes.byref(d))
    if rc < 0:
        _check(rc)
    return rc


def conv2d_value_tile(d):
    """The tile (TILE_*) ALGO_AUTO runs d in on float32 values; 0 if bitsliced."""
    rc = lib().hobflops_conv2d_value_tile(ctypes.byref(d))
    if rc < 0:
        _check(rc)
    return rc


def conv2d_on_values(ifm, w, d, tile, out=None):
    """conv2d on float32 values in the given tile (TILE_*), whichever kernel
    ALGO_AUTO would pick: the same results."""
    out = _conv_out(ifm, w, d, out)
    _call(ifm.device, lib().hobflops_conv2d_on_values, _ptr(ifm), _ptr(w), _ptr(out), ctypes.byref(d),
          tile)
    return out


def muladd(a, b, c, n, in_fmt, acc_fmt, out=None, round=ROUND_NEAREST_EVEN):
    """Element-wise add(widen(c), mul(a, b)) on flat planes of n elements."""
    in_fmt, acc_fmt = fmt(in_fmt), fmt(acc_fmt)
    if out is None:
        out = torch.empty(plane_shape(1, n, acc_fmt), dtype=torch.int32, device=a.device)
    for t, name in ((a, "a"), (b, "b"), (c, "c")):
        _require(t, 4 * plane_words(1, n, in_fmt), f"muladd {name}")
    _require(out, 4 * plane_words(1, n, acc_fmt), "muladd out")
    _call(a.device, lib().hobflops_muladd, _ptr(a), _ptr(b), _ptr(c), _ptr(out), n, in_fmt, acc_fmt,
          round)
    return out


def muladd_supported(in_fmt, acc_fmt, round=ROUND_NEAREST_EVEN):
    return bool(lib().hobflops_muladd_supported(fmt(in_fmt), fmt(acc_fmt), round))


def netlist_ops(in_fmt, acc_fmt, round=ROUND_NEAREST_EVEN):
    """dict of VALU ops per 32-lane word: conv 'mac' (fused step), 'mul' and 'accum'
    (the split kernel's two roles), element-wise 'muladd'; 0 where not generated."""
    v = [ctypes.c_int() for _ in range(4)]
    rc = lib().hobflops_netlist_ops(fmt(in_fmt), fmt(acc_fmt), round,
                                    *[ctypes.byref(x) for x in v])
    if rc != 0:
        raise HobflopsError(rc, lib().hobflops_status_string(rc).decode())
    return dict(zip(("mac", "mul", "accum", "muladd"), (x.value for x in v)))


def avgpool(planes, N, H, W, C, in_fmt, acc_fmt, out_fmt, out=None, round=ROUND_NEAREST_EVEN):
    """Global average pooling: planes [N*H*W, ceil(C/32), NB_in] -> [N, ceil(C/32), NB_out]."""
    in_fmt, acc_fmt, out_fmt = fmt(in_fmt), fmt(acc_fmt), fmt(out_fmt)
    if out is None:
        out = torch.empty(plane_shape(N, C, out_fmt), dtype=torch.int32, device=planes.device)
    if N > 0 and H > 0 and W > 0 and C > 0:
        _require(planes, 4 * plane_words(N * H * W, C, in_fmt), "avgpool planes")
        _require(out, 4 * plane_words(N, C, out_fmt), "avgpool out")
    _call(planes.device, lib().hobflops_avgpool, _ptr(planes), _ptr(out), N, H, W, C, in_fmt, acc_fmt,
          out_fmt, round)
    return out


def avgpool_supported(in_fmt, acc_fmt, out_fmt, round=ROUND_NEAREST_EVEN):
    return bool(lib().hobflops_avgpool_supported(fmt(in_fmt), fmt(acc_fmt), fmt(out_fmt), round))


def avgpool_netlist_ops(in_fmt, acc_fmt, out_fmt, round=ROUND_NEAREST_EVEN):
    """dict of VALU ops per 32-lane word of the pooling netlists: 'accum', 'scale'."""
    v = [ctypes.c_int() for _ in range(2)]
    rc = lib().hobflops_avgpool_netlist_ops(fmt(in_fmt), fmt(acc_fmt), fmt(out_fmt), round,
                                            *[ctypes.byref(x) for x in v])
    if rc != 0:
        raise HobflopsError(rc, lib().hobflops_status_string(rc).decode())
    return dict(zip(("accum", "scale"), (x.value for x in v)))


def wait_failures(reset=True):
    """Give-ups of the split kernel's bounded waits on the current device since
    the last reset (synchronises the device); nonzero means some launch's
    results are invalid."""
    n = ctypes.c_uint32()
    _check(lib().hobflops_wait_failures(ctypes.byref(n), 1 if reset else 0))
    return n.value


def set_wait_limit(sleeps):
    """Bound, in sleeps, of every counter wait in later split-kernel launches
    (process-wide; 0 gives up at the first look that misses)."""
    _check(lib().hobflops_set_wait_limit(int(sleeps)))


def get_wait_limit():
    return int(lib().hobflops_get_wait_limit())


# ---- blocks of narrow floats and the gated feed-forward block ------------------
# The launches go to the current stream of the first tensor's device.


def _rows(t, name):
    """(pointer, rows, columns, elements between rows) of a GPU matrix whose rows are dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("hobflops operates on GPU tensors only")
    if t.dim() != 2:
        raise ValueError(f"{name}: a matrix is needed, not {tuple(t.shape)}")
    r, c = t.shape
    if t.is_contiguous():
        return t.data_ptr(), r, c, c
    sr, sc = t.stride()
    if (c > 1 and sc != 1) or (r > 1 and sr < c):
        raise ValueError(f"{name}: rows must be dense and not overlap")
    return t.data_ptr(), r, c, (sr if r > 1 else c)


def _type(t, name):
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name}: float32, bfloat16 or float16 values are needed, not {t.dtype}")
    return kind


def _dense(t, shape, dtype, device, name):
    """The pointer of a dense tensor of this shape, type and device."""
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise TypeError(f"{name}: a tensor on {device} is needed")
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor {tuple(shape)} is needed")
    return t.data_ptr()


def _out_rows(t, shape, dtype, device, name):
    """(output matrix, pointer, elements between rows): a caller's, with dense rows, or a new one."""
    if t is None:
        t = torch.empty(shape, dtype=dtype, device=device)
        return t, t.data_ptr(), shape[1]
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name}: a {dtype} tensor {tuple(shape)} on {device} is needed")
    ptr, _, _, ld = _rows(t, name)
    return t, ptr, ld


def block_shapes(rows, cols, f, group=32):
    """The shapes of the codes and of the scales of a [rows, cols] matrix in blocks."""
    bits = 1 + sum(f) if isinstance(f, tuple) else 1 + f.wE + f.wF
    return (rows, (cols * bits + 7) // 8), (rows, -(-cols // group))


def _block_shapes(rows, cols, f, group):
    # a group that the library refuses: nothing to size, the call reports it
    return block_shapes(rows, cols, f, group) if group in (32, 64, 128) else ((0, 0), (0, 0))


def block_pack(src, f, group=32, scale=SCALE_POW2, codes=None, scales=None):
    """float32, bfloat16 or float16 values [rows, cols] (dense rows, any distance apart) -> codes
    of the narrow format f ((4, 3), (5, 2): 8 bits, (2, 1): 4 bits), uint8, and the scales of
    their groups: (codes, scales). 8-bit codes take groups of 32 and SCALE_POW2."""
    f = fmt(f)
    ptr, rows, cols, ld = _rows(src, "block_pack src")
    kind = _type(src, "block_pack src")
    cshape, sshape = _block_shapes(rows, cols, f, group)
    stype, dev = _SCALE_TYPES.get(scale, torch.uint8), src.device
    if codes is None:
        codes = torch.empty(cshape, dtype=torch.uint8, device=dev)
        pc = codes.data_ptr()
    else:
        pc = _dense(codes, cshape, torch.uint8, dev, "block_pack codes")
    if scales is None:
        scales = torch.empty(sshape, dtype=stype, device=dev)
        ps = scales.data_ptr()
    else:
        ps = _dense(scales, sshape, stype, dev, "block_pack scales")
    _call(dev, lib().hobflops_block_pack, ptr, kind, rows, cols, ld, f, group, scale, pc, ps)
    return codes, scales


def block_unpack(codes, scales, cols, f, group=32, dtype=torch.float32, out=None):
    """Codes and scales of block_pack -> the values they stand for, [rows, cols]."""
    f = fmt(f)
    if not isinstance(codes, torch.Tensor) or not codes.is_cuda or codes.dim() != 2:
        raise TypeError("block_unpack: codes [rows, bytes] on a GPU are needed")
    rows, dev = codes.shape[0], codes.device
    cshape, sshape = _block_shapes(rows, cols, f, group)
    if scales.dtype not in _SCALES:
        raise TypeError(f"block_unpack: scales of {scales.dtype}")
    pc = _dense(codes, cshape, torch.uint8, dev, "block_unpack codes")
    ps = _dense(scales, sshape, scales.dtype, dev, "block_unpack scales")
    if out is not None:
        dtype = out.dtype
    out, ptr, ld = _out_rows(out, (rows, cols), dtype, dev, "block_unpack out")
    _call(dev, lib().hobflops_block_unpack, pc, ps, rows, cols, f, group, _SCALES[scales.dtype], ptr,
          _type(out, "block_unpack out"), ld)
    return out


def _gated_weights(x, w_gate, w_up):
    """(pointers, F, D, row distance) of the two weights."""
    pg, F, D, ldw = _rows(w_gate, "gated w_gate")
    pu, Fu, Du, ldu = _rows(w_up, "gated w_up")
    if (Fu, Du) != (F, D) or ldu != ldw:
        raise ValueError("gated: w_gate and w_up must have one shape and row distance")
    if w_gate.dtype != x.dtype or w_up.dtype != x.dtype:
        raise TypeError("gated: the weights must have the type of the activations")
    if w_gate.device != x.device or w_up.device != x.device:
        raise TypeError("gated: tensors of different devices")
    return pg, pu, F, D, ldw


def _align(*ptrs):
    """The alignment in bytes that all the pointers have: 2, 4, 8 or 16."""
    bits = 16
    for p in ptrs:
        bits |= p
    return bits & -bits


def _no_gradient(name, *tensors):
    """Says that autograd records nothing of a call whose inputs it follows."""
    if torch.is_grad_enabled() and any(t.requires_grad for t in tensors):
        warnings.warn(f"{name}: its result carries no gradient to its inputs; wrap it in a "
                      "torch.autograd.Function (gated_backward has the gated block's gradients), or "
                      "call it under torch.no_grad()", stacklevel=3)


def _workspace(d, backward, device):
    n = ctypes.c_int64()
    _check(lib().hobflops_gated_workspace(ctypes.byref(d), backward, ctypes.byref(n)))
    if n.value == 0:
        return None, 0, 0
    ws = torch.empty(n.value, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), n.value


def gated_forward(x, w_gate, w_up, act=GATE_SILU, ckpt=None, out=None):
    """h = act(x w_gate^T) * (x w_up^T): x [T, D], w_gate and w_up [F, D], bfloat16 or float16 ->
    h [T, F]. With ckpt, an 8-bit format: (h, saved), the blocks of x, g and u in that format, for
    gated_backward. Autograd records nothing of it."""
    px, T, D, ldx = _rows(x, "gated_forward x")
    pg, pu, F, Dw, ldw = _gated_weights(x, w_gate, w_up)
    if Dw != D:
        raise ValueError("gated_forward: x and the weights differ in D")
    _no_gradient("gated_forward", x, w_gate, w_up)
    h, ph, ldh = _out_rows(out, (T, F), x.dtype, x.device, "gated_forward out")
    f = Fmt(0, 0) if ckpt is None else fmt(ckpt)
    d = GatedDesc(T, D, F, ldx, ldw, ldh, _type(x, "gated_forward x"), act, f,
                  _align(px, pg, pu))
    ws, pw, nw = _workspace(d, 0, x.device)
    forward = lib().hobflops_gated_forward
    if ckpt is None:
        _call(x.device, forward, ctypes.byref(d), px, pg, pu, ph, None, None, None, None, pw, nw)
        return h
    cshape, sshape = block_shapes(T, F, f)
    blocks = [torch.empty(s, dtype=torch.uint8, device=x.device)
              for s in (cshape, sshape, cshape, sshape)]
    _call(x.device, forward, ctypes.byref(d), px, pg, pu, ph, *[b.data_ptr() for b in blocks], pw, nw)
    return h, GatedSaved(block_pack(x, f), tuple(blocks[:2]), tuple(blocks[2:]), f)


def gated_backward(dh, saved, w_gate, w_up, act=GATE_SILU):
    """The gradients (dx, dw_gate, dw_up) of gated_forward from dh [T, F] and what it saved."""
    ph, T, F, ldh = _rows(dh, "gated_backward dh")
    pg, pu, Fw, D, ldw = _gated_weights(dh, w_gate, w_up)
    if Fw != F:
        raise ValueError("gated_backward: dh and the weights differ in F")
    f = saved.fmt
    dev, dtype = dh.device, dh.dtype
    ptrs = []
    for (codes, scales), cols, name in ((saved.x, D, "x"), (saved.gate, F, "gate"),
                                        (saved.up, F, "up")):
        cshape, sshape = block_shapes(T, cols, f)
        ptrs += [_dense(codes, cshape, torch.uint8, dev, f"gated_backward saved.{name} codes"),
                 _dense(scales, sshape, torch.uint8, dev, f"gated_backward saved.{name} scales")]
    d = GatedDesc(T, D, F, D, ldw, ldh, _type(dh, "gated_backward dh"), act, f, _align(pg, pu))
    ws, pw, nw = _workspace(d, 1, dev)
    dx = torch.empty((T, D), dtype=dtype, device=dev)
    dw_gate = torch.empty((F, D), dtype=dtype, device=dev)
    dw_up = torch.empty((F, D), dtype=dtype, device=dev)
    _call(dev, lib().hobflops_gated_backward, ctypes.byref(d), ph, *ptrs, pg, pu, dx.data_ptr(),
          dw_gate.data_ptr(), dw_up.data_ptr(), pw, nw)
    return dx, dw_gate, dw_up


def _w4(x, weights, group, out, name):
    """Checked arguments of a product with 4-bit weights: the output, and what comes before and
    after the activation."""
    px, T, K, ldx = _rows(x, name)
    dev, scale = x.device, weights[1].dtype
    if scale not in _SCALES:
        raise TypeError(f"{name}: scales of {scale}")
    if group not in (32, 64, 128):
        raise ValueError(f"{name}: groups of 32, 64 or 128 are supported, not {group}")
    N = weights[0].shape[0]
    cshape, sshape = (N, (K + 1) // 2), (N, -(-K // group))
    ptrs = [_dense(w, sshape if i & 1 else cshape, scale if i & 1 else torch.uint8, dev, name)
            for i, w in enumerate(weights)]
    y, py, ldy = _out_rows(out, (T, N), x.dtype, dev, name)
    return (y, (px, _type(x, name), T, K, N, ldx, *ptrs, group, _SCALES[scale]),
            (py, ldy))


def w4_linear(x, codes, scales, group=32, out=None):
    """y = x W^T for few tokens: x [T, K] bfloat16 or float16, W [N, K] as 4-bit codes and scales
    (block_pack with the format (2, 1)) -> y [T, N]."""
    y, head, tail = _w4(x, (codes, scales), group, out, "w4_linear")
    _no_gradient("w4_linear", x)
    _call(x.device, lib().hobflops_w4_linear, *head, *tail)
    return y


def w4_gated(x, g_codes, g_scales, u_codes, u_scales, act=GATE_SILU, group=32, out=None):
    """h = act(x Wg^T) * (x Wu^T) for few tokens, both weights as 4-bit codes and scales."""
    y, head, tail = _w4(x, (g_codes, g_scales, u_codes, u_scales), group, out, "w4_gated")
    _no_gradient("w4_gated", x)
    _call(x.device, lib().hobflops_w4_gated, *head, act, *tail)
    return y

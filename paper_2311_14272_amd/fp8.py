"""Layers in 8 bits: binding of crisp_fp8_* (include/crisp_fp8.h).  Argument marshalling only, every step runs in the HIP
kernels.

A matrix in 8 bits (Fp8Mat) is e4m3 values with one fp32 scale for each block of 128 columns of a row (ROWS, activations and
gradients) or of 128 x 128 elements (TILES, weights).  One layer's training step is

    x8, x_t = quantize_both(x)                   # x: T x K
    w8, w_t = quantize_both(W, TILES, mask=...)  # W: S x K, after each change of W; mask: pruned positions count as zero
    y = product(x8, w8)                          # T x S
    dx, dw = linear_backward(dy, x_t, w_t)       # T x K and S x K, dw in fp32: the gradient crisp_select_mask and adamw take

and serving is y = linear(x, w8).  Tensors live on the current device; work goes to the current stream.

Autograd does not see these calls: a result carries no gradient, also where an argument requires one, and linear_backward is
called by hand.  A bias's gradient, the sum of dy's rows, is not among its results.
"""
from __future__ import annotations

import ctypes as C
import struct
from functools import lru_cache

import torch

from . import crisp

ROWS, TILES = 0, 1
BLOCK = 128
_IN = {torch.float32: 0, torch.bfloat16: 1}     # CRISP_IN_*, and the CRISP_Y_* of the same types
CODES = (torch.float8_e4m3fn, torch.uint8)      # what holds e4m3 codes: other 8-bit formats have other values for the same byte


class _Mat(C.Structure):
    _fields_ = [("q", C.c_void_p), ("scale", C.c_void_p), ("ld", C.c_int64), ("lds", C.c_int64), ("rows", C.c_int64),
                ("cols", C.c_int64), ("kind", C.c_int32), ("reserved", C.c_int32)]


_pack = struct.Struct("@PPqqqqii").pack          # a crisp_fp8_mat as bytes: a third of the time of a ctypes structure

_pack_ep = struct.Struct("@PPPqii").pack         # and a crisp_epilogue

_lib = None
_device = torch._C._cuda_getDevice


def lib():
    global _lib
    if _lib is None:
        L = crisp.lib()
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        mat = ep = C.c_void_p       # bytes (Fp8Mat.c) or a pointer to a structure
        L.crisp_fp8_quant.argtypes = [vp, i32, i64, i64, i64, vp, mat, mat, vp]
        L.crisp_fp8_product.argtypes = [mat, mat, vp, i64, i32, ep, vp]
        L.crisp_fp8_linear.argtypes = [vp, i32, i64, i64, mat, vp, i64, i32, ep, vp, C.c_size_t, vp]
        L.crisp_fp8_linear_backward.argtypes = [vp, i32, i64, i64, i64, mat, mat, vp, i64, i32, vp, i64, i32, i32, vp, C.c_size_t, vp]
        for f in (L.crisp_fp8_quant, L.crisp_fp8_product, L.crisp_fp8_linear, L.crisp_fp8_linear_backward):
            f.restype = i32
        for f in (L.crisp_fp8_linear_ws, L.crisp_fp8_linear_backward_ws):
            f.argtypes, f.restype = [i64, i64], C.c_size_t
        _lib = L
    return _lib


@lru_cache(maxsize=1024)
def _linear_ws(T, K):
    return lib().crisp_fp8_linear_ws(T, K)


@lru_cache(maxsize=1024)
def _backward_ws(T, S):
    return lib().crisp_fp8_linear_backward_ws(T, S)


def _here(t, what):
    """A tensor's address; it has to be on the device whose stream the work goes to."""
    if t.get_device() != _device():              # (-1 for a tensor of the host)
        raise ValueError("%s is on %s, not on the current GPU" % (what, t.device))
    return t.data_ptr()


def _workspace(ws):
    """(address, bytes) of a caller's workspace: bytes one behind the other."""
    if not ws.is_contiguous():
        raise ValueError("ws is not contiguous")
    return _here(ws, "ws"), ws.numel() * ws.element_size()


def _mats_here(*mats):
    now = _device()
    for m in mats:
        if m is not None and m.dev != now:
            raise ValueError("a matrix is on GPU %d, not on the current one" % m.dev)


def _blocks(n):
    return -(-n // BLOCK)


class Fp8Mat:
    """A rows x cols matrix in 8 bits over existing tensors: q, rows x at least round_up(cols, 128) bytes (uint8 or
    float8_e4m3fn, zeros behind the columns), and scale, fp32, ceil(cols/128) x rows (ROWS) or ceil(rows/128) x ceil(cols/128)
    (TILES); both with contiguous rows, any row stride that the header allows.  Keeps the tensors alive."""
    __slots__ = ("q", "scale", "rows", "cols", "kind", "c", "dev")

    def __init__(self, q, scale, rows, cols, kind):
        if kind not in (ROWS, TILES):
            raise ValueError("kind is ROWS or TILES")
        want = (_blocks(cols), rows) if kind == ROWS else (_blocks(rows), _blocks(cols))
        if q.dtype not in CODES or q.dim() != 2 or q.shape[0] != rows or q.shape[1] < _blocks(cols) * BLOCK or q.stride(1) != 1:
            raise ValueError("q: %d rows of at least %d e4m3 codes (float8_e4m3fn or uint8), each row contiguous" % (rows, _blocks(cols) * BLOCK))
        if scale.dtype != torch.float32 or scale.dim() != 2 or tuple(scale.shape) != want or (scale.stride(1) != 1 and want[1] > 1):
            raise ValueError("scale: %d x %d fp32, each row contiguous" % want)
        self._fill(q, scale, rows, cols, kind)

    def _fill(self, q, scale, rows, cols, kind):
        self.q, self.scale, self.rows, self.cols, self.kind, self.dev = q, scale, rows, cols, kind, q.get_device()
        # (a tensor of one row may carry any row stride)
        self.c = _pack(_here(q, "q"), _here(scale, "scale"), q.stride(0) if rows > 1 else max(q.stride(0), q.shape[1]),
                       scale.stride(0) if scale.shape[0] > 1 else max(scale.stride(0), scale.shape[1]), rows, cols, kind, 0)


def _new(rows, cols, kind, device):
    b = (cols + 127) >> 7
    out = Fp8Mat.__new__(Fp8Mat)
    out.q = q = torch.empty_strided((rows, b << 7), (b << 7, 1), dtype=torch.float8_e4m3fn, device=device)      # (0.4 us less than empty)
    shape = (b, rows) if kind == ROWS else ((rows + 127) >> 7, b)
    out.scale = scale = torch.empty_strided(shape, (shape[1], 1), dtype=torch.float32, device=device)
    out.rows, out.cols, out.kind, out.dev = rows, cols, kind, q.get_device()
    out.c = _pack(q.data_ptr(), scale.data_ptr(), b << 7, shape[1], rows, cols, kind, 0)
    return out


def alloc_mat(rows, cols, kind=ROWS, device="cuda") -> Fp8Mat:
    """Buffers of a rows x cols matrix in 8 bits, to be filled by quantize."""
    if kind not in (ROWS, TILES) or rows < 1 or cols < 1:
        raise ValueError("a matrix of at least 1 x 1, kind ROWS or TILES")
    out = _new(rows, cols, kind, device)
    _here(out.q, "the matrix")
    return out


def _input(x):
    """(address, type, rows, cols, row stride) of a matrix with contiguous rows."""
    if x.dim() != 2 or x.dtype not in _IN or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("a matrix of fp32 or bf16 with contiguous rows is wanted")
    rows, cols = x.shape
    if rows < 1 or cols < 1:
        raise ValueError("a matrix of at least 1 x 1 is wanted")
    return _here(x, "input"), _IN[x.dtype], rows, cols, x.stride(0) if rows > 1 else max(x.stride(0), cols)


def _quant(x, mask, out, out_t, inp=None, kind=None):
    p, t, rows, cols, ldx = inp or _input(x)
    _mats_here(out, out_t)
    if kind is not None and ((out is not None and out.kind != kind) or (out_t is not None and out_t.kind != kind)):
        raise ValueError("out has another kind of scales")
    if mask is not None:
        if mask.dtype != torch.int32 or not mask.is_contiguous() or mask.numel() < rows * (-(-cols // 32)):
            raise ValueError("mask: rows x ceil(cols/32) contiguous int32 words")
        mask = _here(mask, "mask")
    st = (_lib or lib()).crisp_fp8_quant(p, t, rows, cols, ldx, mask, out and out.c, out_t and out_t.c, crisp._stream())
    if st != crisp.OK:
        raise crisp.CrispError("crisp_fp8_quant", st)


def quantize(x, kind=ROWS, mask=None, out=None) -> Fp8Mat:
    """crisp_fp8_quant of x (fp32 or bf16) into out, allocated when not given.  mask: words as crisp.DeviceLayer.nm_mask or
    adamw.hybrid_mask hold them; positions whose bit is not set count as zero."""
    inp = _input(x)
    if out is None:
        out = _new(inp[2], inp[3], kind, x.device)
    _quant(x, mask, out, None, inp, kind)
    return out


def quantize_both(x, kind=ROWS, mask=None, out=None, out_t=None):
    """(x, its transpose) in 8 bits, in one pass over x."""
    inp = _input(x)
    if out is None:
        out = _new(inp[2], inp[3], kind, x.device)
    if out_t is None:
        out_t = _new(inp[3], inp[2], kind, x.device)
    _quant(x, mask, out, out_t, inp, kind)
    return out, out_t


def _output(T, S, out, out_dtype, device, what="out"):
    """(the result's tensor, its address, its row stride)"""
    if out is None:
        out = torch.empty_strided((T, S), (S, 1), dtype=out_dtype, device=device)
        return out, out.data_ptr(), S
    if out.dtype not in _IN or tuple(out.shape) != (T, S) or (S > 1 and out.stride(1) != 1):
        raise ValueError("%s: %d x %d of fp32 or bf16 with contiguous rows" % (what, T, S))
    return out, _here(out, what), out.stride(0) if T > 1 else max(out.stride(0), S)


def _epilogue(ep, bias, S):
    """What the library takes: NULL, or a structure."""
    if bias is None:
        return None if ep is None else C.byref(ep)
    if ep is not None:
        raise ValueError("bias goes into the epilogue when there is one")
    if bias.dtype != torch.float32 or bias.dim() != 1 or bias.numel() != S or (S > 1 and bias.stride(0) != 1):
        raise ValueError("bias: %d contiguous fp32 values" % S)
    return _pack_ep(0, _here(bias, "bias"), 0, 0, 0, 0)


def product(x: Fp8Mat, w: Fp8Mat, out=None, out_dtype=torch.bfloat16, bias=None, ep=None):
    """crisp_fp8_product: x w^T, x.rows x w.rows; into out, allocated as out_dtype when not given.  ep: crisp.epilogue(...),
    per column of the result."""
    _mats_here(x, w)
    out, to, ldy = _output(x.rows, w.rows, out, out_dtype, x.q.device)
    ep = _epilogue(ep, bias, w.rows)
    st = (_lib or lib()).crisp_fp8_product(x.c, w.c, to, ldy, _IN[out.dtype], ep, crisp._stream())
    if st != crisp.OK:
        raise crisp.CrispError("crisp_fp8_product", st)
    return out


def linear(x, w: Fp8Mat, out=None, out_dtype=torch.bfloat16, bias=None, ep=None, ws=None):
    """crisp_fp8_linear: the layer for activations x (T x K, fp32 or bf16).  ws: a workspace of the caller's (contiguous,
    crisp_fp8_linear_ws bytes); allocated for the call when not given."""
    p, kind, T, K, ldx = _input(x)
    if K != w.cols:
        raise ValueError("x has %d columns, the weights %d" % (K, w.cols))
    _mats_here(w)
    out, to, ldy = _output(T, w.rows, out, out_dtype, x.device)
    if ep is not None or bias is not None:
        ep = _epilogue(ep, bias, w.rows)
    if ws is None:
        room = _linear_ws(T, K)
        at = None
        if room:
            ws = torch.empty_strided((room,), (1,), dtype=torch.uint8, device=x.device)
            at = ws.data_ptr()
    else:
        at, room = _workspace(ws)
    st = (_lib or lib()).crisp_fp8_linear(p, kind, T, ldx, w.c, to, ldy, _IN[out.dtype], ep, at, room, crisp._stream())
    if st != crisp.OK:
        raise crisp.CrispError("crisp_fp8_linear", st)
    return out


def linear_backward(dy, x_t: Fp8Mat, w_t: Fp8Mat, dx=None, dw=None, accumulate=False, ws=None):
    """crisp_fp8_linear_backward, the gradients of y = linear(x, w): (dx, dw) from dy (T x S, fp32 or bf16), x_t = x^T in 8 bits
    (K x T) and w_t = W^T in 8 bits (K x S); x_t or w_t None: that gradient (dw or dx) is not computed.  dx is T x K, bf16 unless
    given; dw is S x K, fp32 unless given.  accumulate: dw (given) += the gradient.  ws: as in linear
    (crisp_fp8_linear_backward_ws bytes)."""
    p, kind, T, S, ldg = _input(dy)
    if (x_t is not None and x_t.cols != T) or (w_t is not None and w_t.cols != S):
        raise ValueError("dy is %d x %d, x^T has %s columns, W^T %s" % (T, S, x_t and x_t.cols, w_t and w_t.cols))
    if (accumulate and dw is None) or (dx is not None and w_t is None) or (dw is not None and x_t is None):
        raise ValueError("accumulate adds to a dw that is given; dx needs w_t, dw needs x_t")
    _mats_here(x_t, w_t)
    L = _lib or lib()
    to_x = to_w = None
    ldx = ldw = tx = tw = 0
    if w_t is not None:
        dx, to_x, ldx = _output(T, w_t.rows, dx, torch.bfloat16, dy.device, "dx")
        tx = _IN[dx.dtype]
    if x_t is not None:
        dw, to_w, ldw = _output(S, x_t.rows, dw, torch.float32, dy.device, "dw")
        tw = _IN[dw.dtype]
    if ws is None:
        room = max(16, _backward_ws(T, S))
        ws = torch.empty_strided((room,), (1,), dtype=torch.uint8, device=dy.device)
        at = ws.data_ptr()
    else:
        at, room = _workspace(ws)
    st = L.crisp_fp8_linear_backward(p, kind, T, S, ldg, x_t and x_t.c, w_t and w_t.c, to_x, ldx, tx, to_w, ldw, tw, int(accumulate),
                                     at, room, crisp._stream())
    if st != crisp.OK:
        raise crisp.CrispError("crisp_fp8_linear_backward", st)
    return dx, dw

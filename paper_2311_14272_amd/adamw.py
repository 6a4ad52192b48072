"""The optimiser step of fine-tuning: binding of crisp_adamw_batch and crisp_hybrid_mask (include/crisp_adamw.h).  Argument
marshalling only, every step runs in the HIP kernels.

    tensors = [adamw.tensor(w, g, m, v, mask=..., row_len=K, weight_decay=0.01), ...]
    batch = adamw.make_batch(tensors)             # once, as long as the buffers stay where they are
    adamw.step(batch, lr=1e-4, step=t)            # all tensors

Moments are fp32 tensors, or e4m3 ones (torch.float8_e4m3fn or uint8) with a scale for each 128 elements (m_scale, v_scale);
alloc_moments makes either.  Tensors live on the current device; work goes to the current stream.

Autograd does not see a step: weights change in place and keep their version, so a graph that was recorded before the step must
not be run backward after it.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import crisp
from .fp8 import CODES, _here

BLOCK = 128
_P = {torch.float32: 0, torch.bfloat16: 1}      # CRISP_P_*


class _Tensor(C.Structure):
    _fields_ = [("w", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("w_copy", C.c_void_p), ("mask", C.c_void_p), ("numel", C.c_int64), ("row_len", C.c_int64),
                ("w_type", C.c_int32), ("g_type", C.c_int32), ("moments", C.c_int32), ("weight_decay", C.c_float)]


class _Hyper(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("grad_scale", C.c_double),
                ("step", C.c_int64), ("live", C.c_void_p)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        L = crisp.lib()
        vp = C.c_void_p
        L.crisp_adamw_batch.argtypes = [C.c_int32, C.POINTER(_Tensor), C.POINTER(_Hyper), vp]
        L.crisp_hybrid_mask.argtypes = [C.POINTER(crisp.LayerDesc), vp, vp, vp, vp, vp]
        L.crisp_adamw_batch.restype = L.crisp_hybrid_mask.restype = C.c_int32
        _lib = L
    return _lib


def alloc_moments(numel, bits=32, device="cuda") -> dict:
    """Moments before the first step, as keyword arguments of tensor()."""
    if bits == 32:
        return {k: torch.zeros(numel, dtype=torch.float32, device=device) for k in ("m", "v")}
    if bits != 8:
        raise ValueError("moments are held in 32 or in 8 bits")
    out = {k: torch.zeros(numel, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for k in ("m", "v")}
    return out | {k: torch.zeros(-(-numel // BLOCK), dtype=torch.float32, device=device) for k in ("m_scale", "v_scale")}


def tensor(w, g, m, v, m_scale=None, v_scale=None, w_copy=None, mask=None, row_len=0, weight_decay=0.0) -> dict:
    """One tensor of a step; see crisp_adamw_tensor.  All contiguous; mask: int32 words of numel/row_len rows."""
    n = w.numel()
    eight = m_scale is not None or v_scale is not None
    if w.dtype not in _P or g.dtype not in _P:
        raise ValueError("weights and gradients are fp32 or bf16")
    if g.numel() != n or m.numel() != n or v.numel() != n or (w_copy is not None and w_copy.numel() != n):
        raise ValueError("weights, gradients and moments are of one size")
    if eight and (m_scale is None or v_scale is None or m.dtype not in CODES or v.dtype not in CODES
                  or any(s.dtype != torch.float32 or s.numel() != -(-n // BLOCK) for s in (m_scale, v_scale))):
        raise ValueError("8-bit moments: e4m3 codes (float8_e4m3fn or uint8), and an fp32 scale for each %d elements in m_scale and v_scale" % BLOCK)
    if not eight and (m.dtype != torch.float32 or v.dtype != torch.float32):
        raise ValueError("moments without scales are fp32")
    if w_copy is not None and (w_copy.element_size() != 2 or w_copy.dtype not in (torch.bfloat16, torch.int16) or w.dtype != torch.float32):
        raise ValueError("w_copy: bf16, of fp32 weights")
    if mask is not None and (row_len < 1 or n % row_len or mask.dtype != torch.int32 or mask.numel() < n // row_len * -(-row_len // 32)):
        raise ValueError("mask: ceil(row_len/32) int32 words for each of the numel/row_len rows")
    every = {"w": w, "g": g, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale, "w_copy": w_copy, "mask": mask}
    for k, t in every.items():
        if t is not None and not t.is_contiguous():
            raise ValueError("%s is not contiguous" % k)
    return every | {"row_len": row_len, "weight_decay": weight_decay}


class Batch:
    """The tensors of a step as the library takes them; keeps them alive."""

    def __init__(self, tensors):
        if not tensors:
            raise ValueError("no tensors")
        self.tensors = tensors
        self.c = (_Tensor * len(tensors))()
        for c, t in zip(self.c, tensors):
            for k in ("w", "g", "m", "v", "m_scale", "v_scale", "w_copy", "mask"):
                setattr(c, k, None if t[k] is None else _here(t[k], k))
            c.numel, c.row_len = t["w"].numel(), t["row_len"]
            c.w_type, c.g_type = _P[t["w"].dtype], _P[t["g"].dtype]
            c.moments, c.weight_decay = int(t["m_scale"] is not None), t["weight_decay"]
        starts = [p for c in self.c if c.numel for p in (c.w, c.m, c.v, c.m_scale, c.v_scale, c.w_copy) if p]
        if len(set(starts)) != len(starts):
            raise ValueError("a tensor, or a buffer that a step writes, comes twice")
        self.device = tensors[0]["w"].device


def make_batch(tensors) -> Batch:
    """The argument array of crisp_adamw_batch for tensor(...)s, built once."""
    return Batch(tensors)


def live(lr, step, grad_scale=1.0, skip=False, device="cuda"):
    """The values of a step on the device (crisp_adamw_live), as an int32 tensor for step(live=...) and set_live."""
    out = torch.empty(4, dtype=torch.int32, device=device)
    set_live(out, lr, step, grad_scale, skip)
    return out


def set_live(out, lr, step, grad_scale=1.0, skip=False):
    """Writes new values; ordered on the current stream like any other work."""
    two = torch.tensor([lr, grad_scale], dtype=torch.float32).view(torch.int32)
    out.copy_(torch.cat([two, torch.tensor([step, int(skip)], dtype=torch.int32)]))


def step(batch: Batch, lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, step=1, grad_scale=1.0, live=None):
    """crisp_adamw_batch: one step of all tensors, in place.  live: see live(); lr, step and grad_scale are then its."""
    if batch.device.index != torch._C._cuda_getDevice():
        raise ValueError("the tensors are on %s, not on the current GPU" % batch.device)
    if live is not None and (live.dtype != torch.int32 or live.numel() != 4 or not live.is_contiguous()):
        raise ValueError("live: four int32 words, as live() makes them")
    h = _Hyper(lr, beta1, beta2, eps, grad_scale, step, None if live is None else _here(live, "live"))
    st = lib().crisp_adamw_batch(len(batch.c), batch.c, C.byref(h), crisp._stream())
    if st != crisp.OK:
        raise crisp.CrispError("crisp_adamw_batch", st)


def hybrid_mask(layer: crisp.DeviceLayer, out=None):
    """crisp_hybrid_mask of a pruned layer: its N:M bits inside its kept blocks, for tensor(mask=...) and fp8.quantize."""
    out = torch.empty_like(layer.nm_mask) if out is None else out
    if out.dtype != torch.int32 or not out.is_contiguous() or out.numel() < layer.sizes.mask_words:
        raise ValueError("out: %d contiguous int32 words" % layer.sizes.mask_words)
    st = lib().crisp_hybrid_mask(C.byref(layer.desc), _here(layer.nm_mask, "nm_mask"), _here(layer.row_ptr, "row_ptr"),
                                 _here(layer.col_idx, "col_idx"), _here(out, "out"), crisp._stream())
    if st != crisp.OK:
        raise crisp.CrispError("crisp_hybrid_mask", st)
    return out

"""Plain NumPy forms of the 8-bit quantiser, product and optimiser step, written from their formulas: fp32 where the
definition names a rounding, fp64 elsewhere."""
import numpy as np

F = np.float32
LEAST = F(2.0 ** -126)


def e4m3(x):
    """x rounded to the nearest e4m3 value (ties to even), |x| <= 464; NaN and infinities become NaN."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        e = np.maximum(np.floor(np.log2(np.where(x == 0, 1.0, np.abs(x)))), -6.0)
        step = np.exp2(np.where(np.isfinite(e), e, 0.0) - 3.0)
        y = np.rint(x / step) * step
        return np.where(np.isfinite(x) & (np.abs(y) <= 448.0), y, np.nan)


def scale_of(amax):
    with np.errstate(all="ignore"):
        s = (amax.astype(F) / F(448.0)).astype(F)
        return np.where(s < LEAST, LEAST, s)       # (a NaN stays)


def _codes(x, s):
    with np.errstate(all="ignore"):
        return e4m3((x.astype(F) * (F(1.0) / s).astype(F)).astype(F))


def _amax(a, axis):
    return np.max(np.abs(a), axis=axis)            # NaN propagates


def quant(x, tiles, mask=None):
    """(values the codes stand for without scale, R x round_up(C,128); scales in the library's layout)."""
    x = np.asarray(x, dtype=F)
    if mask is not None:
        x = np.where(mask, x, F(0))
    R, C = x.shape
    Rb, Cb = -(-R // 128), -(-C // 128)
    full = np.zeros((Rb * 128, Cb * 128), dtype=F)
    full[:R, :C] = x
    if tiles:
        s = scale_of(_amax(full.reshape(Rb, 128, Cb, 128), (1, 3)))
        return _codes(full, np.repeat(np.repeat(s, 128, 0), 128, 1))[:R], s
    s = scale_of(_amax(full.reshape(Rb * 128, Cb, 128), 2))
    return _codes(full, np.repeat(s, 128, 1))[:R], np.ascontiguousarray(s[:R].T)


def held(q, s, tiles):
    """fp64 values of a matrix in 8 bits."""
    R = q.shape[0]
    each = np.repeat(np.repeat(s, 128, 0), 128, 1)[:R] if tiles else np.repeat(s.T, 128, 1)
    with np.errstate(all="ignore"):
        return q.astype(np.float64) * each.astype(np.float64)


def product_bound(A, K):
    """|error| of the fp32 sums where A = |x| |w|^T: at most 128 roundings (of up to a whole step, 2^-23) inside a block's sum;
    the product of the scales, the product with it and the additions of the blocks, half a step each."""
    nb = -(-K // 128)
    return (128 * 2.0 ** -23 + (nb + 3) * 2.0 ** -24) * A


def product_bound_fast(A, K):
    """The same where the 8-bit matrix instruction adds: it sums groups of eight products, aligned to the largest one's exponent
    with 13 bits kept below it; each of the seven others loses less than 2^-13 of the largest one's power of two,
    which is at most that product's magnitude, which the group's sum of magnitudes bounds: 7 * 2^-13 of it."""
    return product_bound(A, K) + 7 * 2.0 ** -13 * A


def bits_of(mask_rows):
    """int32 words of a truth matrix, bit k % 32 of word k // 32."""
    R, C = mask_rows.shape
    full = np.zeros((R, -(-C // 32) * 32), dtype=np.uint64)
    full[:, :C] = mask_rows
    words = (full.reshape(R, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return words.astype(np.uint32).view(np.int32)


def bf16(x):
    """fp32 values rounded to bf16, as fp32."""
    b = np.asarray(x, dtype=F).view(np.uint32).astype(np.uint64)
    return (((b + 0x7FFF + ((b >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(F)


def adamw(w, g, m, v, keep, lr, b1, b2, eps, gs, step, decay, scales=None, w_bf16=False):
    """The step in fp32, operation by operation.  scales: (m's, v's) of 8-bit moments, m and v then hold code values.
    Returns (w, m, v, new scales or None)."""
    w, g, m, v = (np.asarray(a, dtype=F) for a in (w, g, m, v))
    n = w.size
    decay = float(F(decay))
    with np.errstate(all="ignore"):
        if scales is not None:
            ms, vs = (np.repeat(np.asarray(s, dtype=F), 128)[:n] for s in scales)
            m, u = m * ms, v * vs
            v = u * u
        g1 = g * F(gs)
        m1 = F(b1) * m + F(1.0 - b1) * g1
        v1 = F(b2) * v + F(1.0 - b2) * (g1 * g1)
        u = np.sqrt(v1)
        d = u * F(1.0 / np.sqrt(1.0 - b2 ** step)) + F(eps)
        new = w * F(1.0 - lr * decay) - F(lr / (1.0 - b1 ** step)) * (m1 / d)
    if keep is not None:
        new, m1, v1, u = np.where(keep, new, w), np.where(keep, m1, F(0)), np.where(keep, v1, F(0)), np.where(keep, u, F(0))
    assert all(a.dtype == F for a in (new, m1, v1, u))
    if w_bf16:
        new = bf16(new) if keep is None else np.where(keep, bf16(new), w)
    if scales is None:
        return new, m1, v1, None
    pad = -(-n // 128) * 128
    mf, uf = np.zeros(pad, dtype=F), np.zeros(pad, dtype=F)
    mf[:n], uf[:n] = m1, u
    ns = [scale_of(_amax(a.reshape(-1, 128), 1)) for a in (mf, uf)]
    qm = _codes(mf, np.repeat(ns[0], 128))
    with np.errstate(all="ignore"):
        q = (uf * (F(1.0) / np.repeat(ns[1], 128)).astype(F)).astype(F)
    q = np.where((uf > 0) & (q < F(2.0 ** -9)), F(2.0 ** -9), q)
    return new, qm[:n].astype(F), e4m3(q)[:n].astype(F), ns

"""The 8-bit layers and the optimiser step where no GPU is needed: exported names, struct layouts, refusals before any device
call, and the plain forms that the GPU tests compare with."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2311_14272_amd import adamw, crisp, fp8

import lowbit_util as U

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000     # never dereferenced: the calls below fail their checks first


def _declared(header):
    text = open(os.path.join(ROOT, "include", header)).read()
    return sorted(set(re.findall(r"CRISP_API[^;(]*?\b(crisp_\w+)\s*\(", text)))


def test_headers_and_exports():
    assert _declared("crisp_fp8.h") == ["crisp_fp8_linear", "crisp_fp8_linear_backward", "crisp_fp8_linear_backward_ws", "crisp_fp8_linear_ws",
                                         "crisp_fp8_product", "crisp_fp8_quant"]
    assert _declared("crisp_adamw.h") == ["crisp_adamw_batch", "crisp_hybrid_mask"]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "crisp_fp8.h"\n#include "crisp_adamw.h"\nint main(void) {' \
          'printf("%zu %zu %zu %zu %zu %zu %zu\\n", sizeof(crisp_fp8_mat), offsetof(crisp_fp8_mat, kind), sizeof(crisp_adamw_tensor),' \
          ' offsetof(crisp_adamw_tensor, weight_decay), sizeof(crisp_adamw_hyper), offsetof(crisp_adamw_hyper, live),' \
          ' sizeof(crisp_adamw_live)); return 0; }'
    exe = "/tmp/crisp_lowbit_layout"
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-x", "c", "-", "-o", exe],
                       input=src, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(fp8._Mat), fp8._Mat.kind.offset, C.sizeof(adamw._Tensor), adamw._Tensor.weight_decay.offset,
                   C.sizeof(adamw._Hyper), adamw._Hyper.live.offset, 16]
    for name in _declared("crisp_fp8.h") + _declared("crisp_adamw.h"):
        assert getattr(crisp.lib(), name) is not None


def _mat(R, cols_, kind_=fp8.ROWS, **k):
    b = -(-cols_ // 128)
    m = dict(q=FAKE, scale=FAKE, ld=b * 128, lds=R if kind_ == fp8.ROWS else b, rows=R, cols=cols_, kind=kind_, reserved=0)
    m.update(k)
    return fp8._Mat(**m)


def _quant(rows=8, cols=200, X=FAKE, t=1, ldx=None, mask=None, Q="", Qt=None):
    Q = _mat(rows, cols) if Q == "" else Q
    return fp8.lib().crisp_fp8_quant(X, t, rows, cols, cols if ldx is None else ldx, mask, C.byref(Q) if Q else None,
                                     C.byref(Qt) if Qt else None, None)


def test_quant_refusals():
    assert _quant(Q=None) == crisp.EINVAL
    assert _quant(X=None) == crisp.EINVAL
    assert _quant(t=2) == crisp.EINVAL
    assert _quant(ldx=199) == crisp.ESHAPE
    assert _quant(rows=0, Q=_mat(1, 200)) == crisp.ESHAPE
    assert _quant(cols=0, Q=_mat(8, 1)) == crisp.ESHAPE
    assert _quant(X=FAKE + 1) == crisp.EALIGN
    assert _quant(X=FAKE + 2, t=0) == crisp.EALIGN
    assert _quant(mask=FAKE + 2) == crisp.EALIGN
    for bad, status in ((dict(q=None), crisp.EINVAL), (dict(scale=None), crisp.EINVAL), (dict(kind=2), crisp.EINVAL),
                        (dict(reserved=1), crisp.EINVAL), (dict(ld=200), crisp.ESHAPE), (dict(ld=264), crisp.EALIGN),
                        (dict(lds=7), crisp.ESHAPE), (dict(q=FAKE + 8), crisp.EALIGN), (dict(scale=FAKE + 2), crisp.EALIGN),
                        (dict(rows=9, lds=9), crisp.ESHAPE), (dict(cols=201), crisp.ESHAPE), (dict(rows=-1), crisp.ESHAPE),
                        (dict(ld=1 << 31), crisp.ESHAPE)):
        assert _quant(Q=_mat(8, 200, **bad)) == status, bad
    assert _quant(Qt=_mat(8, 200)) == crisp.ESHAPE                       # not the transpose
    assert _quant(Qt=_mat(200, 8, fp8.TILES)) == crisp.EINVAL            # another kind
    assert _quant(rows=1 << 27, cols=512, Q=_mat(1 << 27, 512)) == crisp.ESHAPE     # 2^29 blocks of a row


def test_two_results_in_one_place_are_refused():
    """A square matrix and its transpose, or a layer's two gradients, cannot go to the same buffer: which of the two stayed would be chance."""
    at = lambda q, scale: _mat(256, 256, q=FAKE * q, scale=FAKE * scale)
    for Qt in (at(1, 7), at(7, 1), at(1, 1)):
        assert _quant(rows=256, cols=256, Q=at(1, 1), Qt=Qt) == crisp.EINVAL
    L = fp8.lib()
    m, need = _mat(256, 256), L.crisp_fp8_linear_backward_ws(256, 256)
    assert L.crisp_fp8_linear_backward(FAKE, 1, 256, 256, 256, C.byref(m), C.byref(m), 64 * FAKE, 256, 0, 64 * FAKE, 256, 0, 0, FAKE, need, None) == crisp.EINVAL


def _product(X=None, W=None, Y=FAKE, ldy=64, t=1, ep=None):
    X, W = X or _mat(16, 256), W or _mat(64, 256, fp8.TILES)
    return fp8.lib().crisp_fp8_product(C.byref(X), C.byref(W), Y, ldy, t, C.byref(ep) if ep else None, None)


def test_product_refusals():
    assert _product(Y=None) == crisp.EINVAL
    assert _product(t=2) == crisp.EINVAL
    assert _product(X=_mat(16, 256, fp8.TILES)) == crisp.EINVAL          # X has a scale for each row
    assert _product(W=_mat(64, 255, fp8.TILES)) == crisp.ESHAPE
    assert _product(ldy=63) == crisp.ESHAPE
    assert _product(Y=FAKE + 1) == crisp.EALIGN
    assert _product(Y=FAKE + 2, t=0) == crisp.EALIGN
    assert _product(ep=crisp.Epilogue(None, None, None, 0, 2, 0)) == crisp.EINVAL
    assert _product(ep=crisp.Epilogue(None, None, FAKE, 63, 0, 0)) == crisp.ESHAPE
    assert _product(ep=crisp.Epilogue(None, None, FAKE, 72, 0, 0)) == crisp.ESHAPE      # Y itself with another row length
    assert _product(ep=crisp.Epilogue(FAKE + 2, None, None, 0, 0, 0)) == crisp.EALIGN
    assert _product(X=_mat(1 << 20, 256), W=_mat(1 << 20, 256, fp8.TILES), ldy=1 << 20) == crisp.ESHAPE   # 2^32 tiles
    L = fp8.lib()
    assert L.crisp_fp8_product(None, None, FAKE, 64, 1, None, None) == crisp.EINVAL


def test_linear_refusals():
    L = fp8.lib()
    need = L.crisp_fp8_linear_ws(70, 200)
    assert need == 70 * (256 + 2 * 4)
    assert L.crisp_fp8_linear_ws(16, 200) == 0 and L.crisp_fp8_linear_ws(16, 1025) == 16 * 9 * 132       # one launch up to 128 blocks
    assert L.crisp_fp8_linear_ws(0, 200) == 0 and L.crisp_fp8_linear_ws(16, -1) == 0 and L.crisp_fp8_linear_ws(1 << 27, 512) == 0
    W = _mat(64, 200, fp8.TILES)

    def linear(X=FAKE, t=1, T=70, ldx=200, Y=FAKE, ldy=64, ws=FAKE, n=need):
        return L.crisp_fp8_linear(X, t, T, ldx, C.byref(W), Y, ldy, 1, None, ws, n, None)
    assert linear(X=None) == crisp.EINVAL and linear(Y=None) == crisp.EINVAL and linear(t=7) == crisp.EINVAL
    assert linear(T=0) == crisp.ESHAPE and linear(ldx=199) == crisp.ESHAPE and linear(ldy=63) == crisp.ESHAPE
    assert linear(ws=FAKE + 8) == crisp.EALIGN
    assert linear(ws=None) == crisp.EBUFSIZE and linear(n=need - 1) == crisp.EBUFSIZE
    assert L.crisp_fp8_linear(FAKE, 1, 16, 200, None, FAKE, 64, 1, None, FAKE, need, None) == crisp.EINVAL


def test_linear_backward_refusals():
    L = fp8.lib()
    need = L.crisp_fp8_linear_backward_ws(70, 300)
    assert need == (70 * 3 * 132 + 15) // 16 * 16 + 300 * 132 and L.crisp_fp8_linear_backward_ws(0, 5) == 0 and L.crisp_fp8_linear_backward_ws(5, -1) == 0
    Xt, Wt = _mat(200, 70), _mat(200, 300, fp8.TILES)

    def backward(dY=FAKE, t=1, T=70, S=300, ldg=300, Xt=Xt, Wt=Wt, dX=FAKE, lddx=200, dxt=1, dW=FAKE, lddw=200, dwt=0, acc=0, ws=FAKE, n=need):
        return L.crisp_fp8_linear_backward(dY, t, T, S, ldg, C.byref(Xt) if Xt else None, C.byref(Wt) if Wt else None, dX, lddx, dxt,
                                           dW, lddw, dwt, acc, ws, n, None)
    for bad in (dict(dX=None, dW=None), dict(dY=None), dict(t=2), dict(Xt=None), dict(Wt=None), dict(acc=2), dict(dxt=2), dict(dwt=-1),
                dict(Xt=_mat(200, 70, kind=2))):
        assert backward(**bad) == crisp.EINVAL, bad
    for bad in (dict(T=0), dict(S=0), dict(ldg=299), dict(T=71), dict(S=301, ldg=301), dict(Xt=_mat(201, 70)), dict(lddx=199), dict(lddw=199)):
        assert backward(**bad) == crisp.ESHAPE, bad
    for bad in (dict(dY=FAKE + 1), dict(dX=FAKE + 1), dict(dW=FAKE + 2), dict(ws=FAKE + 4)):
        assert backward(**bad) == crisp.EALIGN, bad
    assert backward(ws=None) == crisp.EBUFSIZE and backward(n=need - 1) == crisp.EBUFSIZE


def _adamw(h=None, count=1, **k):
    t = dict(w=FAKE, g=FAKE, m=FAKE, v=FAKE, m_scale=None, v_scale=None, w_copy=None, mask=None, numel=1000, row_len=0, w_type=0,
             g_type=0, moments=0, weight_decay=0.0)
    t.update(k)
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, live=None)
    hyper.update(h or {})
    # the first tensor has no elements, so that nothing would be enqueued for it
    arr = (adamw._Tensor * 2)(adamw._Tensor(**{**t, "numel": 0, "w": None}), adamw._Tensor(**t))
    return adamw.lib().crisp_adamw_batch(count + 1 if count > 0 else count, arr, C.byref(adamw._Hyper(**hyper)), None)


def test_adamw_refusals():
    for k in ("w", "g", "m", "v"):
        assert _adamw(**{k: None}) == crisp.EINVAL
        assert _adamw(**{k: FAKE + 8}) == crisp.EALIGN
    assert _adamw(count=0) == crisp.EINVAL and _adamw(count=1 << 20) == crisp.EINVAL
    for bad in (dict(w_type=2), dict(g_type=-1), dict(moments=2), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
                dict(moments=1), dict(moments=1, m_scale=FAKE), dict(m_scale=FAKE), dict(w_type=1, w_copy=FAKE)):
        assert _adamw(**bad) == crisp.EINVAL, bad
    for bad in (dict(numel=-1), dict(mask=FAKE), dict(mask=FAKE, row_len=300), dict(mask=FAKE, row_len=1, numel=1 << 31),
                dict(numel=1 << 40)):
        assert _adamw(**bad) == crisp.ESHAPE, bad
    assert _adamw(moments=1, m_scale=FAKE + 2, v_scale=FAKE) == crisp.EALIGN
    assert _adamw(mask=FAKE + 1, row_len=10) == crisp.EALIGN and _adamw(w_copy=FAKE + 2) == crisp.EALIGN
    for bad in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(lr=-1.0), dict(lr=float("nan")), dict(step=0),
                dict(step=1 << 31), dict(grad_scale=float("inf"))):
        assert _adamw(h=bad) == crisp.EINVAL, bad
    assert _adamw(h=dict(live=FAKE + 2)) == crisp.EALIGN
    assert adamw.lib().crisp_adamw_batch(1, None, None, None) == crisp.EINVAL


def test_adamw_eps_that_rounds_to_zero():
    """The step divides by the root plus eps in fp32: an eps that is zero there makes NaN of every element without a gradient."""
    h = lambda eps: _adamw(h=dict(eps=eps), numel=0)     # (nothing is enqueued for tensors without elements)
    for bad in (1e-50, 1e-300, 5e-324, 2.0 ** -150):
        assert h(bad) == crisp.EINVAL, bad
    for good in (2.0 ** -149, 1e-40, 1e-8, 1e30):
        assert h(good) == crisp.OK, good


def test_hybrid_mask_refusals():
    L = adamw.lib()
    d = crisp.layer_desc(64, 128, 2, 4, 32, 0.5)
    assert L.crisp_hybrid_mask(C.byref(d), None, FAKE, FAKE, FAKE, None) == crisp.EINVAL
    assert L.crisp_hybrid_mask(C.byref(d), FAKE, FAKE, FAKE, FAKE + 2, None) == crisp.EALIGN
    assert L.crisp_hybrid_mask(None, FAKE, FAKE, FAKE, FAKE, None) == crisp.EINVAL
    assert L.crisp_hybrid_mask(C.byref(crisp.layer_desc(0, 128, 2, 4, 32, 0.5)), FAKE, FAKE, FAKE, FAKE, None) == crisp.ESHAPE


def test_tensors_off_the_gpu_are_refused():
    x = torch.zeros(4, 128)
    with pytest.raises((ValueError, RuntimeError)):      # (without any GPU there is no current one to compare with)
        fp8.Fp8Mat(torch.zeros((4, 128), dtype=torch.uint8), torch.zeros((1, 4)), 4, 128, fp8.ROWS)
    with pytest.raises(ValueError):
        fp8.Fp8Mat(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((1, 4)), 4, 128, fp8.ROWS)
    with pytest.raises(ValueError):
        fp8.quantize(x.to(torch.float64), out=object())
    with pytest.raises(ValueError):
        adamw.tensor(x, x, x, x.double())
    with pytest.raises(ValueError):
        adamw.tensor(x, x, x, x, m_scale=torch.zeros(4))
    with pytest.raises(ValueError):
        adamw.tensor(x.t(), x, x, x)
    with pytest.raises(ValueError):
        adamw.make_batch([])


OTHER_BYTES = [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int8, torch.bool]


@pytest.mark.parametrize("other", OTHER_BYTES, ids=str)
def test_bytes_of_another_type_are_refused(other, monkeypatch):
    """A byte of another format stands for another value: only uint8 (codes) and float8_e4m3fn are taken."""
    monkeypatch.setattr(fp8, "_device", lambda: -1)      # tensors of the host count as on the current device
    scale = torch.zeros((1, 4))
    m = lambda dtype: torch.zeros(4 * 128, dtype=torch.uint8).view(dtype)
    x, s = torch.zeros(4 * 128), torch.zeros(4)
    for good in (torch.uint8, torch.float8_e4m3fn):
        fp8.Fp8Mat(m(good).view(4, 128), scale, 4, 128, fp8.ROWS)
        adamw.tensor(x, x, m(good), m(good), m_scale=s, v_scale=s)
        with pytest.raises(ValueError, match="8-bit moments"):
            adamw.tensor(x, x, m(good), m(other), m_scale=s, v_scale=s)
        with pytest.raises(ValueError, match="8-bit moments"):
            adamw.tensor(x, x, m(other), m(good), m_scale=s, v_scale=s)
    with pytest.raises(ValueError, match="^q: "):
        fp8.Fp8Mat(m(other).view(4, 128), scale, 4, 128, fp8.ROWS)


def test_workspaces_that_are_not_a_row_of_bytes(monkeypatch):
    """A strided workspace has room between its elements that is not the caller's to give, an expanded one has none at all."""
    monkeypatch.setattr(fp8, "_device", lambda: -1)
    monkeypatch.setattr(crisp, "_stream", lambda: None)
    reached = []

    class Library:
        """Takes every call and enqueues nothing."""
        def __getattr__(self, name):
            return lambda *args: reached.append(name) or crisp.OK

    room = max(fp8.lib().crisp_fp8_linear_ws(70, 200), fp8.lib().crisp_fp8_linear_backward_ws(70, 64))
    monkeypatch.setattr(fp8, "_lib", Library())
    codes = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    x, dy = torch.zeros((70, 200)), torch.zeros((70, 64))
    w = fp8.Fp8Mat(codes(64, 256), torch.zeros((2, 64)), 64, 200, fp8.ROWS)
    w_t = fp8.Fp8Mat(codes(200, 128), torch.zeros((1, 200)), 200, 64, fp8.ROWS)
    for good in (codes(room), codes(2, room).view(torch.int16), codes(2, room)[1:]):
        fp8.linear(x, w, ws=good)
        fp8.linear_backward(dy, None, w_t, ws=good)
    assert reached == ["crisp_fp8_linear", "crisp_fp8_linear_backward"] * 3
    for bad in (codes(1).expand(room), codes(2 * room)[::2], codes(room, 2).t()):
        with pytest.raises(ValueError, match="ws"):
            fp8.linear(x, w, ws=bad)
        with pytest.raises(ValueError, match="ws"):
            fp8.linear_backward(dy, None, w_t, ws=bad)


def test_barriers_of_the_product_wait_first():
    """The barrier behind which another wave may overwrite LDS is a bare one: it says nothing about a wave's own reads.  It stands in one
    function only, after the wait for them."""
    csrc = os.path.join(ROOT, "paper_2311_14272_amd", "csrc")
    text = "".join(open(os.path.join(csrc, n)).read() for n in sorted(os.listdir(csrc)) if n.startswith("fp8_"))
    bodies = re.findall(r"__forceinline__ void \w+\(\) \{(.*?)\n\}", text, re.S)
    have = [b for b in bodies if "s_barrier" in b]
    assert len(have) == 1 and text.count("s_barrier") == 1
    assert re.search(r'asm volatile\(""[^;]*"memory"\);.*wait_loads<LEFT>\(\);.*s_barrier\(\);.*asm volatile\(""[^;]*"memory"\);', have[0], re.S)
    wait = next(b for b in bodies if "s_waitcnt" in b)
    assert "LEFT & 15) | 7 << 4 | 0 << 8 |" in wait          # no LDS operation outstanding, however many requests may be


def test_plain_e4m3_rounding():
    """All 256 codes stand for themselves; values between two neighbours go to the nearer one, the middle to the even one."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    fine = codes[np.isfinite(codes)]
    assert fine.max() == 448.0 and (U.e4m3(fine) == fine).all()
    pos = np.unique(fine[fine >= 0])
    mid = (pos[1:] + pos[:-1]) / 2
    even = np.where(np.arange(mid.size) % 2 == 0, pos[:-1], pos[1:])
    assert (U.e4m3(mid) == even).all() and (U.e4m3(-mid) == -even).all()
    assert (U.e4m3(mid * (1 - 1e-9)) == pos[:-1]).all() and (U.e4m3(mid * (1 + 1e-9)) == pos[1:]).all()
    assert U.e4m3(450.0) == 448.0 and np.isnan(U.e4m3(np.nan)) and np.isnan(U.e4m3(np.inf))


def test_plain_step_against_64_bits():
    """The fp32 form of the step that the kernels are held to, against the same formulas in 64 bits.
    In units of 2^-24: m carries the roundings of beta1 (or 1 - beta1), g', the product and the sum, 4; v of 1 - beta2, twice g',
    its square, the product and the sum, 6; the root half of that and its own, 4; the denominator the correction's, the product's,
    the sum's, 7; the quotient 8 and m's 4, on M = |beta1 m| + |(1 - beta1) g'|; the step's rounded size, product and the
    difference 3 more; the weight its factor, product and difference, 3."""
    rng = np.random.default_rng(3)
    n, lr, b1, b2, eps, gs, step, decay = 5000, 1e-3, 0.9, 0.999, 1e-8, 0.25, 7, 0.1
    w, g = rng.normal(size=n).astype(U.F), (rng.normal(size=n) * 10.0 ** rng.uniform(-9, 2, n)).astype(U.F)
    m, v = (rng.normal(size=n) * np.abs(g) * 0.3).astype(U.F), (g * g * rng.uniform(0, 2, n)).astype(U.F)
    nw, nm, nv, _ = U.adamw(w, g, m, v, None, lr, b1, b2, eps, gs, step, decay)
    W, G, M, V = (a.astype(np.float64) for a in (w, g, m, v))
    G = G * gs
    em, ev = b1 * M + (1 - b1) * G, b2 * V + (1 - b2) * G * G
    den = np.sqrt(ev / (1 - b2 ** step)) + eps
    ew = W - lr * decay * W - lr / (1 - b1 ** step) * em / den
    h, tiny = 2.0 ** -24 * 1.01, 1e-44
    size = np.abs(b1 * M) + np.abs((1 - b1) * G)
    assert (np.abs(nm - em) <= 4 * h * size + tiny).all()
    assert (np.abs(nv - ev) <= 6 * h * ev + 4 * tiny).all()
    fine = ev > 1e-36          # (where the second moment is subnormal its roundings are not relative)
    assert (np.abs(nw - ew) <= 3 * h * np.abs(W) + 15 * h * lr / (1 - b1 ** step) * size / den + 1e-30)[fine].all()

"""The 8-bit layers on the GPU against plain forms in fp32 / fp64: codes and scales bit for bit, products within a bound
derived from the order of the roundings."""
import numpy as np
import pytest
import torch

from paper_2311_14272_amd import adamw, crisp, fp8, synth

import lowbit_util as U
import oracle
from gpu_util import dev, host

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().float().cpu().numpy()


def _same(a, b):
    """Equal values, NaN where NaN."""
    return np.array_equal(np.asarray(a, dtype=np.float64), np.asarray(b, dtype=np.float64), equal_nan=True)


def _input(rng, R, C, dtype, stride=0, offset=0):
    """R x C values over many magnitudes, as (device tensor with the row stride and element offset asked for, fp32 values)."""
    x = rng.normal(size=(R, C)) * 10.0 ** rng.uniform(-3, 3, (R, 1)) * np.where(rng.random((R, C)) < 0.01, 50.0, 1.0)
    x[rng.random((R, C)) < 0.05] = 0.0
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    ld = max(C, stride)
    store = torch.zeros(R * ld + offset, dtype=dtype, device="cuda")
    view = store[offset:].view(R, ld)[:, :C]
    view.copy_(t)
    return view, t.float().numpy()


SHAPES = [(1, 1, 0, 0), (1, 128, 0, 0), (3, 127, 0, 0), (5, 129, 0, 0), (128, 128, 0, 0), (129, 257, 0, 0), (200, 64, 72, 0),
          (131, 384, 392, 8), (77, 300, 301, 1), (17, 1000, 0, 3), (260, 512, 0, 0)]


@pytest.mark.parametrize("kind", [fp8.ROWS, fp8.TILES])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_quantize(shape, dtype, kind):
    R, C, stride, offset = shape
    print("quantize", shape, dtype, kind, flush=True)
    rng = np.random.default_rng(R * 1000 + C)
    x, xh = _input(rng, R, C, dtype, stride, offset)
    keep = rng.random((R, C)) < 0.5
    mask = torch.from_numpy(U.bits_of(keep)).cuda()
    for m, k in ((None, None), (mask, keep)):
        q, s = U.quant(xh, kind == fp8.TILES, k)
        qt, st = U.quant(np.ascontiguousarray((xh if k is None else np.where(k, xh, 0)).T), kind == fp8.TILES)
        one = fp8.quantize(x, kind, mask=m)
        a, b = fp8.quantize_both(x, kind, mask=m)
        only_t = fp8.alloc_mat(C, R, kind)
        fp8._quant(x, m, None, only_t)
        for got in (one, a):
            assert _same(_np(got.q), q) and _same(_np(got.scale), s)
        for got in (b, only_t):
            assert _same(_np(got.q), qt) and _same(_np(got.scale), st)


def test_quantize_leaves_what_is_not_its_own():
    """Bytes behind the padded columns, scales behind the last row, and the rows around the matrix stay as they were."""
    R, C = 70, 200
    rng = np.random.default_rng(1)
    x, xh = _input(rng, R, C, torch.bfloat16)
    for kind in (fp8.ROWS, fp8.TILES):
        big = torch.full((R + 2, 272), 0x55, dtype=torch.uint8, device="cuda")
        bigt = torch.full((C + 2, 144), 0x55, dtype=torch.uint8, device="cuda")
        shape, shapet = ((2, R), (1, C)) if kind == fp8.ROWS else ((1, 2), (2, 1))
        sc, sct = (torch.full((s[0] + 2, s[1] + 3), -7.0, device="cuda") for s in (shape, shapet))
        a = fp8.Fp8Mat(big[1:R + 1], sc[1:-1, :-3], R, C, kind)
        b = fp8.Fp8Mat(bigt[1:C + 1], sct[1:-1, :-3], C, R, kind)
        for once in (True, False):
            if once:
                fp8.quantize(x, kind, out=a)
            else:
                fp8.quantize_both(x, kind, out=a, out_t=b)
            q, s = U.quant(xh, kind == fp8.TILES)
            assert _same(big[1:R + 1, :256].view(torch.float8_e4m3fn).float().cpu(), q) and _same(_np(a.scale), s)
            assert (big[0] == 0x55).all() and (big[R + 1] == 0x55).all() and (big[:, 256:] == 0x55).all()
            assert (sc[0] == -7).all() and (sc[-1] == -7).all() and (sc[:, -3:] == -7).all()
        qt, st = U.quant(np.ascontiguousarray(xh.T), kind == fp8.TILES)
        assert _same(bigt[1:C + 1, :128].view(torch.float8_e4m3fn).float().cpu(), qt) and _same(_np(b.scale), st)
        assert (bigt[0] == 0x55).all() and (bigt[C + 1] == 0x55).all() and (bigt[:, 128:] == 0x55).all()
        assert (sct[0] == -7).all() and (sct[-1] == -7).all() and (sct[:, -3:] == -7).all()


@pytest.mark.parametrize("kind", [fp8.ROWS, fp8.TILES])
def test_quantize_extremes(kind):
    """Blocks of zeros, of the smallest and largest numbers, of one infinity, of one NaN; NaN behind a mask is not seen."""
    x = np.zeros((6, 640), dtype=np.float32)
    x[0, :128] = np.linspace(-1, 1, 128) * 1e-44
    x[1, 128:256] = np.float32(3.4e38) * np.linspace(-1, 1, 128, dtype=np.float32)
    x[2, 256:384] = np.arange(128)
    x[2, 300] = np.inf
    x[3, 384:512] = 1.0
    x[3, 400] = np.nan
    x[4, 512:] = -np.inf
    t = torch.from_numpy(x).cuda()
    for src, vals in ((t, x), (t.to(torch.bfloat16), t.to(torch.bfloat16).float().cpu().numpy())):
        a, b = fp8.quantize_both(src, kind)
        for got, v in ((a, vals), (b, np.ascontiguousarray(vals.T)), (fp8.quantize(src, kind), vals)):
            q, s = U.quant(v, kind == fp8.TILES)
            assert _same(_np(got.q), q) and _same(_np(got.scale), s)
        keep = np.isfinite(vals)
        a = fp8.quantize(src, kind, mask=torch.from_numpy(U.bits_of(keep)).cuda())
        q, s = U.quant(vals, kind == fp8.TILES, keep)
        assert _same(_np(a.q), q) and _same(_np(a.scale), s) and np.isfinite(_np(a.q)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_quantize_row_ends(dtype):
    """Rows that end anywhere in a vector, from any address, among NaN: the matrix, its transpose and the layer that quantises
    for itself see the row's own elements only."""
    rng = np.random.default_rng(21)
    for C in [*range(1, 18), *range(121, 137), 260, 389]:
        R, gap, offset = 3 + C % 7, int(rng.integers(1, 9)), int(rng.integers(0, 9))
        x = torch.from_numpy(rng.normal(size=(R, C)).astype(np.float32)).to(dtype)
        store = torch.full((R * (C + gap) + offset,), float("nan"), dtype=dtype, device="cuda")
        view = store[offset:].view(R, C + gap)[:, :C]
        view.copy_(x)
        xh, keep = x.float().numpy(), rng.random((R, C)) < 0.5
        mask = torch.from_numpy(U.bits_of(keep)).cuda()
        for m, k in ((None, None), (mask, keep)):
            a, b = fp8.quantize_both(view, mask=m)
            one = fp8.quantize(view, mask=m)
            q, s = U.quant(xh, False, k)
            qt, st = U.quant(np.ascontiguousarray((xh if k is None else np.where(k, xh, 0)).T), False)
            for got in (a, one):
                assert _same(_np(got.q), q) and _same(_np(got.scale), s), (C, gap, offset)
            assert _same(_np(b.q), qt) and _same(_np(b.scale), st), (C, gap, offset)
        W = fp8.quantize(torch.from_numpy(rng.normal(size=(20, C)).astype(np.float32)).cuda())
        assert torch.equal(fp8.linear(view, W), fp8.product(fp8.quantize(view), W)), (C, gap, offset)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5, 37, 130), (40, 37, 130), (90, 203, 260), (130, 259, 128)], ids=str)
def test_product_into_any_place(shape, dtype):
    """Y at any address and row stride gets the same bits, and nothing around it changes."""
    T, S, K = shape
    X, W, _, _ = _pair(S, T, S, K, True)
    want = fp8.product(X, W, out_dtype=dtype)
    for offset, gap in ((1, 0), (3, 1), (8, 2), (5, 8 - S % 8), (0, 7)):
        store = torch.full((T * (S + gap) + offset + 9,), -3.0, dtype=dtype, device="cuda")
        rows = store[offset:offset + T * (S + gap)].view(T, S + gap)
        fp8.product(X, W, out=rows[:, :S])
        assert torch.equal(rows[:, :S], want)
        assert (rows[:, S:] == -3).all() and (store[:offset] == -3).all() and (store[offset + T * (S + gap):] == -3).all()


# ---- products ---------------------------------------------------------------------------------------------------

def _pair(seed, T, S, K, w_tiles):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(T, K)) * 10.0 ** rng.uniform(-2, 2, (T, 1))
    w = rng.normal(size=(S, K)) * np.sqrt(2.0 / K)
    X = fp8.quantize(torch.from_numpy(x.astype(np.float32)).cuda(), fp8.ROWS)
    W = fp8.quantize(torch.from_numpy(w.astype(np.float32)).cuda(), fp8.TILES if w_tiles else fp8.ROWS)
    xv, wv = U.held(_np(X.q), _np(X.scale), False), U.held(_np(W.q), _np(W.scale), w_tiles)
    return X, W, xv @ wv.T, np.abs(xv) @ np.abs(wv).T


PRODUCTS = [(1, 1, 1), (1, 16, 128), (2, 48, 100), (1, 1000, 4096), (5, 130, 640), (16, 128, 1152), (17, 33, 257), (31, 520, 2050),
            (48, 64, 8192), (64, 4096, 256), (65, 200, 384), (100, 129, 1000), (128, 128, 128), (129, 300, 512), (255, 257, 300),
            (256, 256, 256), (333, 1000, 130), (512, 512, 1152), (700, 384, 2304), (1030, 1025, 140),
            (3400, 3841, 260), (4096, 4096, 128), (20, 60, 9000), (1000, 40, 300), (90, 70, 200), (1100, 2000, 384),
            (2100, 2050, 200), (65, 65, 65), (80, 96, 1000), (1280, 3456, 130), (1270, 3400, 390), (2300, 4900, 130), (67, 8475, 2879), (265, 9836, 554),
            (195, 8281, 1074), (4947, 1409, 258), (5530, 919, 386), (4267, 2690, 130), (1864, 7758, 261),
            (24, 9000, 300), (9000, 24, 300), (20, 3000, 4200), (3000, 20, 4200), (30, 700, 1000), (16, 12000, 1100)]


@pytest.mark.parametrize("w_tiles", [True, False], ids=["tiles", "rows"])
@pytest.mark.parametrize("shape", PRODUCTS, ids=str)
def test_product(shape, w_tiles):
    T, S, K = shape
    print("product", shape, w_tiles, flush=True)
    X, W, Y, A = _pair(T + S + K, T, S, K, w_tiles)
    bound = U.product_bound(A, K)
    y32 = fp8.product(X, W, out_dtype=torch.float32)
    err = np.abs(_np(y32) - Y)
    assert (err <= bound + 1e-37).all(), float((err / (bound + 1e-37)).max())
    y16 = fp8.product(X, W)
    fast = U.product_bound_fast(A, K)
    err = np.abs(_np(y16) - Y)
    assert (err <= fast + 2.0 ** -8 * (np.abs(Y) + fast) + 1e-37).all(), float((err / (fast + 2.0 ** -8 * np.abs(Y) + 1e-37)).max())
    # into rows longer than the result and behind other memory; what lies around it stays
    for dtype, ld, at in ((torch.float32, S + 5, 1), (torch.bfloat16, (S + 15) // 8 * 8, 8), (torch.bfloat16, S + 1, 1)):
        store = torch.full((T * ld + 2 * ld + at,), -3.0, dtype=dtype, device="cuda")
        out = store[at:at + T * ld].view(T, ld)[:, :S]
        fp8.product(X, W, out)
        assert torch.equal(out, (y32 if dtype == torch.float32 else y16))
        rest = torch.ones_like(store, dtype=torch.bool)
        rest[at:at + T * ld].view(T, ld)[:, :S] = False
        assert (store[rest] == -3.0).all()


@pytest.mark.parametrize("shape", [(3, 40, 200), (40, 250, 300), (300, 136, 513), (512, 768, 256)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_product_epilogue(shape, dtype):
    """Scale, bias, residual and ReLU, each one fp32 operation on the sum: exactly the plain product's sums put through them.
    A residual that is Y itself accumulates."""
    T, S, K = shape
    X, W, Y, A = _pair(7 * T + S, T, S, K, True)
    y = fp8.product(X, W, out_dtype=torch.float32)
    fast = dtype == torch.bfloat16          # sums of another instruction, seen through one rounding: held to its bound
    g = torch.Generator(device="cuda").manual_seed(5)
    sc, bi = (torch.randn(S, generator=g, device="cuda") for _ in range(2))
    res = torch.randn((T, S + 3), generator=g, device="cuda").to(dtype)

    def check(got, want, factor):
        assert got.dtype == dtype
        if not fast:
            assert torch.equal(got, want)
            return
        # the two sums differ by at most both bounds, times the scale; then at most three fp32 roundings of either and one to bf16
        far = torch.from_numpy(U.product_bound_fast(A, K) + U.product_bound(A, K)).cuda() * abs(factor)
        big = want.double().abs() + far + bi.double().abs() + res[:, :S].double().abs()
        assert ((got.double() - want.double()).abs() <= far + (2.0 ** -8 + 6 * 2.0 ** -24) * big).all()

    for relu in (False, True):
        for use in range(8):
            ep = crisp.epilogue(sc if use & 1 else None, bi if use & 2 else None, res if use & 4 else None, S + 3, relu)
            want = y
            want = want * sc if use & 1 else want
            want = want + bi if use & 2 else want
            want = want + res[:, :S].float() if use & 4 else want
            want = want.clamp(min=0) if relu else want
            check(fp8.product(X, W, out_dtype=dtype, ep=ep), want, (sc if use & 1 else 1.0))
    check(fp8.product(X, W, out_dtype=dtype, bias=bi), y + bi, 1.0)
    acc = res.clone()
    fp8.product(X, W, acc[:, :S], ep=crisp.epilogue(residual=acc, ldr=S + 3))
    check(acc[:, :S], y + res[:, :S].float(), 1.0)
    assert torch.equal(acc[:, S:], res[:, S:])


def test_product_keeps_rows_apart():
    """A NaN or an infinity in one row of X or W reaches that row's or column's results and no other; rows with a large ld."""
    T, S, K = 150, 140, 400
    rng = np.random.default_rng(2)
    x, w = rng.normal(size=(T, K)).astype(np.float32), rng.normal(size=(S, K)).astype(np.float32)
    clean = fp8.product(fp8.quantize(torch.from_numpy(x).cuda()), fp8.quantize(torch.from_numpy(w).cuda()), out_dtype=torch.float32)
    x[77, 3], x[149, 399], w[20, 130] = np.nan, np.inf, -np.inf
    X = fp8.Fp8Mat(torch.zeros((T, 528), dtype=torch.uint8, device="cuda"), torch.zeros((4, T + 9), device="cuda")[:, :T], T, K, fp8.ROWS)
    fp8.quantize(torch.from_numpy(x).cuda(), out=X)
    y = fp8.product(X, fp8.quantize(torch.from_numpy(w).cuda()), out_dtype=torch.float32)
    bad = torch.zeros((T, S), dtype=torch.bool, device="cuda")
    bad[77], bad[149], bad[:, 20] = True, True, True
    assert y[bad].isnan().all() and torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 40, 200), (20, 70, 3000), (150, 140, 400), (2300, 4900, 130)], ids=str)
def test_relu_lets_nan_through(shape, dtype):
    """A NaN or an infinity in a block makes NaN of the results that use it, behind a ReLU too; the others are as without them."""
    T, S, K = shape
    rng = np.random.default_rng(T)
    x, w = rng.normal(size=(T, K)).astype(np.float32), rng.normal(size=(S, K)).astype(np.float32)
    ep = crisp.epilogue(relu=True)
    q = lambda a: fp8.quantize(torch.from_numpy(a).cuda())
    clean = fp8.product(q(x), q(w), out_dtype=dtype)
    assert torch.equal(fp8.product(q(x), q(w), out_dtype=dtype, ep=ep), clean.clamp(min=0))
    x[1, 3], x[T - 1, K - 1], w[20, 7] = np.nan, np.inf, -np.inf
    bad = torch.zeros((T, S), dtype=torch.bool, device="cuda")
    bad[1], bad[T - 1], bad[:, 20] = True, True, True
    for y in (fp8.product(q(x), q(w), out_dtype=dtype, ep=ep), fp8.linear(torch.from_numpy(x).cuda(), q(w), out_dtype=dtype, ep=ep)):
        assert y[bad].isnan().all() and torch.equal(y[~bad], clean[~bad].clamp(min=0))


@pytest.mark.parametrize("shape", [(1, 1, 5), (1, 300, 4096), (2, 64, 256), (4, 513, 1100), (7, 96, 384), (8, 256, 8192), (1, 33, 16384), (1, 50, 16385), (2, 200, 8000), (16, 40, 1024),
                                   (15, 512, 1000), (17, 64, 128), (13, 700, 2050),
                                   (16, 128, 128), (33, 200, 1152), (300, 264, 640)], ids=str)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_linear_is_quantize_and_product(shape, dtype):
    T, S, K = shape
    print("linear", shape, dtype, flush=True)
    rng = np.random.default_rng(T + S + K)
    w = fp8.quantize(torch.from_numpy((rng.normal(size=(S, K)) * 0.05).astype(np.float32)).cuda(), fp8.TILES)
    w_rows = fp8.quantize(torch.from_numpy((rng.normal(size=(S, K)) * 0.05).astype(np.float32)).cuda(), fp8.ROWS)
    bias = torch.randn(S, device="cuda")
    for stride, offset in ((0, 0), (K + 3, 1), ((K + 15) // 8 * 8, 8)):
        x, xh = _input(rng, T, K, dtype, stride, offset)
        x8 = fp8.quantize(x)
        for weights in (w, w_rows):
            assert torch.equal(fp8.linear(x, weights), fp8.product(x8, weights))
            assert torch.equal(fp8.linear(x, weights, out_dtype=torch.float32, bias=bias),
                               fp8.product(x8, weights, out_dtype=torch.float32, bias=bias))


def test_refusals_that_the_binding_makes():
    x = torch.randn((8, 256), device="cuda")
    x8, t8 = fp8.quantize(x), fp8.quantize(x, fp8.TILES)
    for bad in (lambda: fp8.quantize(x, fp8.ROWS, out=t8), lambda: fp8.quantize(x.t()), lambda: fp8.quantize(x[:0]),
                lambda: fp8.quantize(x.half()), lambda: fp8.quantize(x.cpu()), lambda: fp8.linear(x[:, :128], t8),
                lambda: fp8.linear(x, t8, out=torch.empty((8, 9), device="cuda")), lambda: fp8.linear(x, t8, bias=torch.zeros(9, device="cuda")),
                lambda: fp8.linear(x, t8, bias=torch.zeros(8, device="cuda"), ep=crisp.epilogue()),
                lambda: fp8.quantize(x, mask=torch.zeros(63, dtype=torch.int32, device="cuda")),
                lambda: fp8.Fp8Mat(x8.q, x8.scale, 8, 257, fp8.ROWS), lambda: fp8.Fp8Mat(x8.q, x8.scale.t(), 8, 256, fp8.ROWS),
                lambda: fp8.linear_backward(x, None, None, dw=x), lambda: fp8.linear_backward(x, x8, None, accumulate=True)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: fp8.product(t8, x8),                                        # X with scales of tiles
                lambda: fp8.quantize(x[:1].expand(8, 256)),                         # rows that overlap
                lambda: fp8.product(x8, fp8.quantize(x[:, :128].contiguous())),     # another number of columns
                lambda: fp8.quantize(x, out=fp8.alloc_mat(9, 256)), lambda: fp8.linear_backward(x, None, None)):
        with pytest.raises(crisp.CrispError):
            bad()


def test_rows_far_apart_in_many():
    """Row strides of 2^24 and more: more rows than the kernels without staging are chosen for by their number."""
    ld, K = 1 << 24, 200
    q = torch.zeros((70, ld), dtype=torch.uint8, device="cuda")
    x, w = torch.randn((70, K), device="cuda"), torch.randn((90, K), device="cuda")
    far = fp8.Fp8Mat(q, torch.zeros((2, 70), device="cuda"), 70, K, fp8.ROWS)
    fp8.quantize(x, out=far)
    x8 = fp8.quantize(x)
    for kind in (fp8.TILES, fp8.ROWS):
        w8 = fp8.quantize(w, kind)
        A = np.abs(U.held(_np(x8.q), _np(x8.scale), False)) @ np.abs(U.held(_np(w8.q), _np(w8.scale), kind == fp8.TILES)).T
        a, b = (_np(fp8.product(m, w8, out_dtype=torch.float32)).astype(np.float64) for m in (far, x8))
        assert (np.abs(a - b) <= 2 * U.product_bound(A, K)).all()


def test_long_offsets():
    """A matrix whose last rows lie behind 2^31 bytes: quantised, multiplied, and read as a transpose's columns."""
    rows, ld, K = 20, 1 << 27, 256
    q = torch.zeros((rows, ld), dtype=torch.uint8, device="cuda")
    x = torch.randn((rows, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    far = fp8.Fp8Mat(q, torch.zeros((2, rows), device="cuda"), rows, K, fp8.ROWS)
    fp8.quantize(x, out=far)
    near = fp8.quantize(x)
    assert torch.equal(q[:, :K], near.q.view(torch.uint8)) and torch.equal(far.scale, near.scale)
    w = fp8.quantize(torch.randn((300, K), device="cuda"), fp8.TILES)
    want = fp8.product(near, w, out_dtype=torch.float32)
    assert torch.equal(fp8.product(far, w, out_dtype=torch.float32), want)
    assert torch.equal(fp8.product(w_rows := fp8.quantize(torch.ones((3, K), device="cuda")), far), fp8.product(w_rows, near))
    del q, far
    y = torch.zeros((rows, ld), dtype=torch.float32, device="cuda")
    fp8.product(near, w, y[:, :300])
    assert torch.equal(y[:, :300], want) and not y[:, 300:].any()
    assert torch.equal(fp8.linear(y[:, :300], fp8.quantize(torch.ones((5, 300), device="cuda"))),
                       fp8.linear(want, fp8.quantize(torch.ones((5, 300), device="cuda"))))


# ---- the layer's gradients ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("shape", [(1, 130, 260), (40, 128, 256), (200, 300, 140), (513, 256, 129), (260, 640, 384), (1700, 1500, 140), (500, 512, 1152), (1700, 300, 300)], ids=str)
def test_backward(shape):
    T, S, K = shape
    print("backward", shape, flush=True)
    rng = np.random.default_rng(T * S + K)
    x = torch.from_numpy(rng.normal(size=(T, K)).astype(np.float32)).to(torch.bfloat16).cuda()
    w = torch.from_numpy((rng.normal(size=(S, K)) / np.sqrt(K)).astype(np.float32)).cuda()
    dy = torch.from_numpy((rng.normal(size=(T, S)) * 1e-3).astype(np.float32)).to(torch.bfloat16).cuda()
    x8, x_t = fp8.quantize_both(x)
    w8, w_t = fp8.quantize_both(w, fp8.TILES)
    dx32, dw = fp8.linear_backward(dy, x_t, w_t, dx=torch.empty((T, K), device="cuda"))
    dyh = dy.float().cpu().numpy()
    dq, ds = U.quant(dyh, False)
    dqt, dst = U.quant(np.ascontiguousarray(dyh.T), False)
    d, dt = U.held(dq, ds, False)[:, :S], U.held(dqt, dst, False)[:, :T]
    wv = U.held(_np(w_t.q), _np(w_t.scale), True)[:, :S]          # K x S
    xv = U.held(_np(x_t.q), _np(x_t.scale), False)[:, :T]         # K x T
    for got, want, size, k in ((dx32, d @ wv.T, np.abs(d) @ np.abs(wv).T, S), (dw, dt @ xv.T, np.abs(dt) @ np.abs(xv).T, T)):
        err = np.abs(_np(got) - want)
        assert (err <= U.product_bound(size, k) + 1e-37).all()
    # differences: the loss sum(dy * y(x)) over the weights as held is linear in x, so its difference quotient in any
    # direction is the gradient's product with it; likewise in the weights over the activations as held
    dirx, dirw = rng.normal(size=(T, K)), rng.normal(size=(S, K))
    loss = lambda xx, ww, dd: float((dd * (xx @ ww.T)).sum())
    for got, dd, direction, at in ((dx32, d, dirx, 0), (dw, dt.T, dirw, 1)):
        held_x, held_w = xv.T, wv.T
        hi = loss(held_x + (dirx if at == 0 else 0), held_w + (dirw if at else 0), dd)
        lo = loss(held_x - (dirx if at == 0 else 0), held_w - (dirw if at else 0), dd)
        size = np.abs(d) @ np.abs(wv).T if at == 0 else np.abs(dt) @ np.abs(xv).T
        slack = (U.product_bound(size, T if at else S) * np.abs(direction)).sum() + 1e-10 * (abs(hi) + abs(lo))
        assert abs((hi - lo) / 2 - float((_np(got).astype(np.float64) * direction).sum())) <= slack
    # one gradient alone, and the two calls it is made of
    assert torch.equal(fp8.linear_backward(dy, None, w_t, dx=torch.empty((T, K), device="cuda"))[0], dx32)
    none, alone = fp8.linear_backward(dy, x_t, None)
    dy8, dy_t = fp8.quantize_both(dy)
    both = fp8.linear_backward(dy, x_t, w_t)
    assert torch.equal(both[0], fp8.product(dy8, w_t)) and torch.equal(both[1], dw)
    assert none is None and torch.equal(alone, dw) and torch.equal(fp8.product(dy_t, x_t, out_dtype=torch.float32), dw)
    again, acc = fp8.linear_backward(dy, x_t, w_t, dw=dw.clone(), accumulate=True)
    assert torch.equal(acc, dw + dw)
    want, fast = d @ wv.T, U.product_bound_fast(np.abs(d) @ np.abs(wv).T, S)
    assert (np.abs(_np(again) - want) <= fast + 2.0 ** -8 * (np.abs(want) + fast) + 1e-37).all()


def test_streams_and_graph():
    """A training step of a pruned layer on a side stream, eager and captured; replays give the eager step's bits, with other
    work and an eager step between them."""
    T, S, K = 96, 320, 256
    g = torch.Generator(device="cuda").manual_seed(9)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    w0, bias = rnd(S, K) * 0.05, rnd(S)
    x, dy, token = rnd(T, K).to(torch.bfloat16), (rnd(T, S) * 1e-2).to(torch.bfloat16), rnd(3, K).to(torch.bfloat16)
    w = w0.clone()
    mom = adamw.alloc_moments(S * K, 8)
    dw, dx = torch.empty((S, K), device="cuda"), torch.empty((T, K), dtype=torch.bfloat16, device="cuda")
    y, yt = torch.empty((T, S), dtype=torch.bfloat16, device="cuda"), torch.empty((3, S), dtype=torch.bfloat16, device="cuda")
    batch = adamw.make_batch([adamw.tensor(w, dw, weight_decay=0.1, **mom)])
    live = adamw.live(1e-2, 1)
    mats = [fp8.alloc_mat(T, K), fp8.alloc_mat(K, T), fp8.alloc_mat(S, K, fp8.TILES), fp8.alloc_mat(K, S, fp8.TILES)]

    def step():
        fp8.quantize_both(x, out=mats[0], out_t=mats[1])
        fp8.quantize_both(w, fp8.TILES, out=mats[2], out_t=mats[3])
        fp8.product(mats[0], mats[2], y, bias=bias)
        fp8.linear(token, mats[2], yt)
        fp8.linear_backward(dy, mats[1], mats[3], dx, dw)
        adamw.step(batch, live=live)

    state = [w, mom["m"], mom["v"], mom["m_scale"], mom["v_scale"]]
    outs = [y, yt, dx, dw] + state
    bits = lambda t: t.view(torch.uint8) if t.element_size() == 1 else t

    def reset():
        w.copy_(w0)
        for t in state[1:]:
            bits(t).zero_()

    eager = []
    reset()
    for k in range(4):
        adamw.set_live(live, 1e-2 / (k + 1), k + 1)
        step()
        torch.cuda.synchronize()
        eager.append([bits(t).clone() for t in outs])
    assert not torch.equal(eager[0][4], eager[1][4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        reset()
        adamw.set_live(live, 1e-2, 1)
        step()
        side.synchronize()
        assert all(torch.equal(bits(a), b) for a, b in zip(outs, eager[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    reset()
    other = torch.randn(1 << 16, device="cuda")
    for k in range(4):
        adamw.set_live(live, 1e-2 / (k + 1), k + 1)
        for t in (y, yt, dx, dw):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(bits(a), b) for a, b in zip(outs, eager[k])), k
        other = other * 1.0001 + 1.0
        fp8.linear(token, mats[2])
        torch.cuda.synchronize()


def test_prune_and_fine_tune():
    """The operators in the order a user has them: a layer is pruned by its gradient's saliency, its mask put together, the
    masked weights quantised, forward and backward run in 8 bits, the step taken with the mask held, and the layer pruned again
    with the new gradient; every result against the oracle's or the plain forms on the device's own inputs."""
    T, S, K, n, m, B, d = 192, 96, 320, 2, 4, 32, 0.6
    rng = np.random.default_rng(11)
    w32 = torch.from_numpy((rng.normal(size=(S, K)) * 0.1).astype(np.float32)).cuda()
    w16 = w32.to(torch.bfloat16)
    grad = torch.from_numpy(rng.normal(size=(S, K)).astype(np.float32)).cuda()
    x = torch.from_numpy(rng.normal(size=(T, K)).astype(np.float32)).to(torch.bfloat16).cuda()
    dy = torch.from_numpy((rng.normal(size=(T, S)) * 1e-2).astype(np.float32)).to(torch.bfloat16).cuda()
    layer = crisp.alloc_layer(crisp.layer_desc(S, K, n, m, B, d, crisp.SAL_GRAD))
    mom = adamw.alloc_moments(S * K)
    x8, x_t = fp8.quantize_both(x)
    for t in range(3):
        crisp.prune_and_pack(layer, w16, grad)
        mask = adamw.hybrid_mask(layer)
        sel = oracle.select(w16.view(torch.int16).cpu().numpy().view(np.uint16), grad.cpu().numpy(), n, m, B, d, synth.SAL_GRAD)
        keep = np.asarray(sel.mask).reshape(S, K) != 0
        assert (mask.cpu().numpy().reshape(S, -1) == U.bits_of(keep)).all()
        w8, w_t = fp8.quantize_both(w32, fp8.TILES, mask=mask)
        wq, ws = U.quant(w32.cpu().numpy(), True, keep)
        assert _same(_np(w8.q), wq) and _same(_np(w8.scale), ws)
        y = fp8.linear(x, w8, out_dtype=torch.float32)
        xv, wv = U.held(_np(x8.q), _np(x8.scale), False), U.held(wq, ws, True)
        assert (np.abs(_np(y) - xv @ wv.T) <= U.product_bound(np.abs(xv) @ np.abs(wv).T, K) + 1e-37).all()
        dx, dw = fp8.linear_backward(dy, x_t, w_t)
        before = [a.cpu().numpy().reshape(-1) for a in (w32, dw, mom["m"], mom["v"])]
        adamw.step(adamw.make_batch([adamw.tensor(w32, dw, w_copy=w16, mask=mask, row_len=K, weight_decay=0.01, **mom)]), lr=1e-2, step=t + 1)
        want = U.adamw(*before, keep.reshape(-1), 1e-2, 0.9, 0.999, 1e-8, 1.0, t + 1, 0.01)
        for got, ref in zip((w32, mom["m"], mom["v"]), want):
            assert _same(got.cpu().numpy().reshape(-1), ref)
        assert torch.equal(w16, w32.to(torch.bfloat16))
        grad = dw

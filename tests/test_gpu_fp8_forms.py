"""Every kernel of the 8-bit product on contractions that go several times round its blocks in LDS, with and without an epilogue.
The operands are small integers and their scales powers of two, so that every sum is exact in any order and every result has one
right value; tests/test_fp8_ways_cpu.py holds that the sizes below reach every kernel."""
import pytest
import torch

from paper_2311_14272_amd import crisp, fp8

import lowbit_util as U

pytestmark = pytest.mark.gpu

# T, S, K, none of them a multiple of a tile
LONG = [(7, 333, 3931), (25, 700, 3931), (1030, 31, 3931), (9, 5001, 3931), (5, 100, 12635), (20, 333, 12635), (8, 4099, 8283),
        (333, 301, 2651), (5474, 333, 603), (213, 301, 859), (131, 5495, 2907), (5784, 131, 2651), (586, 4951, 859), (397, 4793, 1627),
        (5149, 1157, 859), (709, 5533, 1627), (3085, 2651, 859), (3853, 3141, 859)]
# T, S, K of layers that quantise their activations themselves
RAW = [(3, 301, 3931), (13, 5001, 1100), (1, 77, 12635), (3, 2001, 5300)]
# T, S, K of gradients, for two launches and for one of either kind
GRADIENTS = [(1700, 300, 300), (1301, 1250, 333), (1001, 1130, 700), (2651, 2590, 65), (1800, 2651, 201)]


def _exact(g, rows, K, tiles):
    """A matrix of integers -2 .. 2 with scales 1/2, 1 and 2 behind other memory, and its values in fp64.  A sum of 12635 products is below
    12635 * 4 * 4 and a multiple of 1/4: 20 bits."""
    b = -(-K // 128)
    q = torch.zeros((rows, b * 128 + 16), dtype=torch.float8_e4m3fn, device="cuda")
    q[:, :K] = torch.randint(-2, 3, (rows, K), generator=g, device="cuda").float().to(torch.float8_e4m3fn)
    shape = (-(-rows // 128), b) if tiles else (b, rows)
    s = torch.exp2(torch.randint(-1, 2, (shape[0], shape[1] + 5), generator=g, device="cuda").float())[:, :shape[1]]
    each = s.repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1) if tiles else s.t().repeat_interleave(128, 1)
    return fp8.Fp8Mat(q, s, rows, K, fp8.TILES if tiles else fp8.ROWS), (q[:, :b * 128].double() * each.double())[:, :K]


def _pair(T, S, K, tiles):
    g = torch.Generator(device="cuda").manual_seed(T + S + K)
    X, xv = _exact(g, T, K, False)
    W, wv = _exact(g, S, K, tiles)
    y = (xv @ wv.t().contiguous()).float()
    assert (y.double().abs() * 4 < 2 ** 24).all()
    return g, X, W, y


@pytest.mark.parametrize("tiles", [True, False], ids=["tiles", "rows"])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_long_contraction(shape, tiles):
    print("product", shape, tiles, flush=True)
    T, S, K = shape
    _, X, W, y = _pair(T, S, K, tiles)
    assert torch.equal(fp8.product(X, W, out_dtype=torch.float32), y)
    assert torch.equal(fp8.product(X, W), y.to(torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tiles", [True, False], ids=["tiles", "rows"])
@pytest.mark.parametrize("shape", LONG, ids=str)
def test_epilogue(shape, tiles, dtype):
    """Scale, bias, residual and ReLU, each alone and together, on exact sums: each step is one fp32 operation, so the bits are given.  The
    residual is another matrix of another row length, or Y itself; what lies around Y stays."""
    print("epilogue", shape, tiles, dtype, flush=True)
    T, S, K = shape
    g, X, W, y = _pair(T, S, K, tiles)
    ld = S + 7
    sc, bi = (torch.randn(S, generator=g, device="cuda") for _ in range(2))
    res = torch.randn((T, ld), generator=g, device="cuda").to(dtype)
    r = res[:, :S].float()
    for scale, bias, residual, relu in ((sc, None, None, False), (None, bi, None, False), (None, None, res, False), (None, None, None, True),
                                        (sc, bi, res, True)):
        want = y if scale is None else y * sc
        want = want if bias is None else want + bi
        want = want if residual is None else want + r
        want = want.clamp(min=0) if relu else want
        got = fp8.product(X, W, out_dtype=dtype, ep=crisp.epilogue(scale, bias, residual, ld, relu))
        assert torch.equal(got, want.to(dtype))
    store = torch.full((ld * (T + 2) + 3,), -3.0, dtype=dtype, device="cuda")       # rows of odd lengths from an odd place
    own = store[ld + 3:ld + 3 + ld * T].view(T, ld)
    own.copy_(res)
    kept = store.clone()
    fp8.product(X, W, own[:, :S], ep=crisp.epilogue(sc, bi, own, ld, True))
    assert torch.equal(own[:, :S], (y * sc + bi + r).clamp(min=0).to(dtype))
    own[:, :S] = res[:, :S]
    assert torch.equal(store, kept)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tiles", [True, False], ids=["tiles", "rows"])
@pytest.mark.parametrize("shape", RAW, ids=str)
def test_epilogue_of_a_layer_in_one_launch(shape, tiles, dtype):
    """The bits of the quantiser and the product, whose epilogue the test above holds."""
    print("linear", shape, tiles, dtype, flush=True)
    T, S, K = shape
    g = torch.Generator(device="cuda").manual_seed(S)
    W, _ = _exact(g, S, K, tiles)
    x = torch.randn((T, K + 3), generator=g, device="cuda")[:, :K]
    sc, bi = (torch.randn(S, generator=g, device="cuda") for _ in range(2))
    res = torch.randn((T, S + 7), generator=g, device="cuda").to(dtype)
    for x in (x, x.to(torch.bfloat16)):
        x8 = fp8.quantize(x)
        for ep in (None, crisp.epilogue(None, bi), crisp.epilogue(sc, bi, res, S + 7, True)):
            assert torch.equal(fp8.linear(x, W, out_dtype=dtype, ep=ep), fp8.product(x8, W, out_dtype=dtype, ep=ep))
        a, b = res.clone(), res.clone()
        fp8.linear(x, W, a[:, :S], ep=crisp.epilogue(sc, bi, a, S + 7, True))
        fp8.product(x8, W, b[:, :S], ep=crisp.epilogue(sc, bi, b, S + 7, True))
        assert torch.equal(a, b) and torch.equal(a[:, S:], res[:, S:])


@pytest.mark.parametrize("shape", GRADIENTS, ids=str)
def test_gradients(shape):
    """Both gradients at once are the two products' bits, also when dW is added to what is there and both lie in longer rows."""
    print("gradients", shape, flush=True)
    T, S, K = shape
    g = torch.Generator(device="cuda").manual_seed(T)
    dy = (torch.randn((T, S), generator=g, device="cuda") * 1e-2).to(torch.bfloat16)
    x_t, _ = _exact(g, K, T, False)
    w_t, _ = _exact(g, K, S, True)
    dy8, dy_t = fp8.quantize_both(dy)
    want_x, want_w = fp8.product(dy8, w_t), fp8.product(dy_t, x_t, out_dtype=torch.float32)
    dx, dw = fp8.linear_backward(dy, x_t, w_t)
    assert torch.equal(dx, want_x) and torch.equal(dw, want_w)
    before = torch.randn((S, K + 3), generator=g, device="cuda")
    big_x, big_w = torch.full((T, K + 1), -3.0, dtype=torch.bfloat16, device="cuda"), before.clone()
    fp8.linear_backward(dy, x_t, w_t, big_x[:, :K], big_w[:, :K], accumulate=True)
    assert torch.equal(big_x[:, :K], want_x) and (big_x[:, K:] == -3).all()
    assert torch.equal(big_w[:, :K], want_w + before[:, :K]) and torch.equal(big_w[:, K:], before[:, K:])


@pytest.mark.parametrize("shape", [(5, 48, 512), (40, 300, 1024), (300, 264, 640), (3085, 2651, 256)], ids=str)
def test_what_the_8_bit_instruction_cuts(shape):
    """In each group of eight one product of 2^16 beside seven of 7.03 = 0.88 * 2^-13 of it, which fall to the cut as far as anything can; the
    large ones cancel, so that nothing else hides the loss.  bf16 results stay within the stated share of the magnitudes, fp32 results
    have every product; without the large ones, so have both."""
    T, S, K = shape
    g = torch.Generator(device="cuda").manual_seed(K)
    sign = lambda *size: torch.randint(0, 2, size, generator=g, device="cuda").float() * 2 - 1
    x, w = 3.75 * sign(T, 1).expand(T, K).clone(), 1.875 * sign(S, 1).expand(S, K).clone()      # (a result's small products have one sign)
    alternate = 1.0 - 2.0 * (torch.arange(K // 8, device="cuda") % 2)
    mat = lambda a: fp8.Fp8Mat(a.to(torch.float8_e4m3fn), torch.ones((K // 128, a.shape[0]), device="cuda"), a.shape[0], K, fp8.ROWS)

    def check(fast):
        X, W = mat(x), mat(w)
        want, size = x.double() @ w.double().t().contiguous(), x.double().abs() @ w.double().abs().t().contiguous()
        err = lambda y: (y.double() - want).abs()
        assert (err(fp8.product(X, W, out_dtype=torch.float32)) <= U.product_bound(size, K)).all()
        assert (err(fp8.product(X, W)) <= fast(size, K) + 2.0 ** -8 * (want.abs() + fast(size, K))).all()

    check(U.product_bound)
    x[:, ::8], w[:, ::8] = 256.0, 256.0 * alternate
    check(U.product_bound_fast)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 48, 512), (300, 264, 640), (3085, 2651, 256)], ids=str)
def test_scales_that_multiply_to_a_subnormal(shape, dtype):
    """Scales of 2^-64 to 2^-80 each: their products lie between 2^-128 and 2^-160, and are off by up to half of 2^-149; the results are what
    those leave.  Blocks of zeros, whose scale is 2^-126, stay zeros."""
    T, S, K = shape
    g = torch.Generator(device="cuda").manual_seed(T)
    X, W = (_exact(g, rows, K, False)[0] for rows in (T, S))
    for m in (X, W):
        m.scale.copy_(torch.exp2(-64 - 16 * torch.rand(m.scale.shape, generator=g, device="cuda")))
        m.scale[0], m.q[:, :128] = 2.0 ** -126, torch.zeros((), dtype=torch.float8_e4m3fn, device="cuda")
    k = -(-K // 128) * 128
    q, s = [m.q[:, :k].double() for m in (X, W)], [m.scale.t().double().repeat_interleave(128, 1) for m in (X, W)]
    held = [a * b for a, b in zip(q, s)]
    want, size = held[0] @ held[1].t().contiguous(), held[0].abs() @ held[1].abs().t().contiguous()
    # a block's sum times the half step of its factor, and half a step of each of the block's additions and of the result; the sums are exact
    slack = 2.0 ** -150 * (q[0].abs() @ q[1].abs().t().contiguous()) + 2.0 ** -150 * (K // 128 + 2) + (K // 128 + 3) * 2.0 ** -24 * size
    y = fp8.product(X, W, out_dtype=dtype).double()
    near = 2.0 ** -8 * (want.abs() + slack) + 2.0 ** -134 if dtype == torch.bfloat16 else 0.0
    assert ((y - want).abs() <= slack + near).all() and want.abs().max() > 2.0 ** -135

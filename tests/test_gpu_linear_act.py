"""The 8-bit linear layer with bias, activation and residual, and its backward pass, against their definitions in 64 bits (fp8_reference.py).

Tolerances.  The sums as in test_gpu_fp8_linear.py: e_z.  The bias adds half a step of fp32.  An activation passes an error of z on by its slope, at most
1.13 (gelu at sqrt 2, its tanh form and silu below that); the activation itself is off by less than 16 half steps of fp32 of its own value
(exponentials of two parts, a reciprocal, a polynomial of degree 9, four products), the tanh form by 6 |v| more, its exponent v being made by three
operations with two constants.  The residual adds a half step of fp32, the output's type one of its own.
The gradient dz is rounded to 16 bits before it is quantised: where its fp32 value lies within its error of a border between two of these numbers
either one is right, and so is what the quantiser makes of either."""
import math

import pytest
import torch

import fp8_reference as ref
from test_gpu_fp8_linear import HALF, TINY, close as close_sums, numbers

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ACTS = [None, "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


def act(z, name):
    """The activation and its slope."""
    if name == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if name == "gelu":
        # (torch.special.ndtr takes 1 + erf: at -10, where this is 7.6e-24, it is 0)
        p = 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        v = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        s = torch.sigmoid(v)
        return z * s, s + z * s * torch.sigmoid(-v) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    return z, torch.ones_like(z)


def act_steps(z, name):
    """Half steps of fp32 that the activation may be off, of its value."""
    if name == "gelu_tanh":
        return 16 + 6 * (2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)).abs()
    return 16.0 if name else 0.0


def stored(X):
    """X in the 8-bit form, rows as add_norm lays them out, with what lies behind the last block of a row set to NaN."""
    num, e, _ = ref.quantize(X)
    rows, cols = X.shape
    blocks = -(-cols // 128)
    q = torch.full((rows, (blocks + 1) * 128), 0x7f, dtype=torch.uint8)
    q[:, :blocks * 128] = 0
    q[:, :cols] = num.to(torch.float8_e4m3fn).view(torch.uint8)
    s = torch.full((rows, (blocks + 3) // 4 * 4), 255, dtype=torch.uint8)
    s[:, :blocks] = (e + 127).to(torch.uint8)
    return q.cuda().view(torch.float8_e4m3fn)[:, :cols], s.cuda()[:, :blocks]


def check(got, want, tol):
    t = got.dtype
    got = got.double().cpu()
    tol = tol + HALF[t] * (want.abs() + tol) + TINY[t]
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / tol).max()))


def forward(slim, n, m, t, x, y, name, bias, residual, keep=True):
    W, X = numbers(n, m, torch.float32, 3) * 0.05, numbers(t, m, torch.bfloat16 if x == "e4m3" else x, 4)
    g = torch.Generator().manual_seed(5)
    b = torch.randn(n, generator=g).to(torch.float32 if bias == "f32" else y) if bias else None
    R = (3 * torch.randn((t, n), generator=g)).to(y) if residual else None
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    Xg = stored(X) if x == "e4m3" else X.cuda()
    Rg = R.cuda() if residual else None
    out = slim.fp8_linear_act(Xg, q, s, None if b is None else b.cuda(), name, Rg, dtype=y, keep=keep)
    Y, Z = out if keep else (out, None)
    assert Y.dtype == y and Y.shape == (t, n)
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    size, z = A.abs() @ B.abs().t(), A @ B.t()
    e = (2 * m / 8 + 16) * 2.0 ** -23 * size
    if t > 16 and y != torch.float32:
        e = e + 2.0 ** -10 * size
    if b is not None:
        z = z + b.double()
        e = e + U * (z.abs() + e)
    if keep:
        check(Z, z, e)
    a, _ = act(z, name)
    e = (1.13 if name else 1.0) * e + act_steps(z, name) * U * a.abs()
    if residual:
        a = a + R.double()
        e = e + U * (a.abs() + e)
    check(Y, a, e)
    return Xg, q, s, b, Rg, Y


@pytest.mark.parametrize("n,m", [(1, 1), (127, 129), (130, 511), (300, 1024), (700, 260)])
@pytest.mark.parametrize("t", [1, 16, 17, 130])
@pytest.mark.parametrize("x,y", [("e4m3", torch.bfloat16), ("e4m3", torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("name,bias,residual", [("gelu", "y", True), ("silu", "f32", False), (None, None, True)])
def test_forward(slim, n, m, t, x, y, name, bias, residual):
    forward(slim, n, m, t, x, y, name, bias, residual)


TILES = [(1024, 512, 1100), (2304, 384, 2100), (1000, 1504, 301), (4096, 1030, 90), (4100, 1030, 70), (520, 9000, 96), (128, 20000, 40), (9000, 700, 16), (4000, 6000, 2100)]


@pytest.mark.parametrize("n,m,t", TILES)
@pytest.mark.parametrize("x,y,name", [("e4m3", torch.float16, "gelu_tanh"), (torch.bfloat16, torch.float32, "silu"), ("e4m3", torch.bfloat16, "relu")])
def test_forward_of_every_tile(slim, n, m, t, x, y, name):
    """Sizes that reach each tile and the parts of a long contraction; the layer's rows and the tokens end inside a tile.  Y in the residual's place."""
    from paper_2405_14917_amd import binding as B
    X, q, s, b, R, Y = forward(slim, n, m, t, x, y, name, "y", True)
    bg, over = b.cuda(), R.clone()
    e = B.SlimEpilogue(bg.data_ptr(), B._DT[y], B.ACTIVATIONS[name], over.data_ptr(), n, None, 0)
    import ctypes
    a = [None, B.F16, t, 0, X[0].data_ptr(), X[0].stride(0), X[1].data_ptr(), X[1].stride(0)] if x == "e4m3" else \
        [X.data_ptr(), B._DT[x], t, m, None, 0, None, 0]
    assert slim.lib.slim_fp8_linear_act(slim.ctx, *a, q.data_ptr(), q.stride(0), s.data_ptr(), s.stride(0), n, m, ctypes.byref(e), over.data_ptr(), B._DT[y],
                                        n) == B.SLIM_OK
    assert torch.equal(over, Y)


@pytest.mark.parametrize("t", [1, 40, 300])
def test_without_an_epilogue_it_is_the_plain_layer(slim, t):
    W, X = numbers(700, 260, torch.float32, 3) * 0.05, numbers(t, 260, torch.bfloat16, 4)
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    for y in (torch.bfloat16, torch.float32):
        want = slim.fp8_linear(X.cuda(), q, s, y)
        assert torch.equal(slim.fp8_linear_act(X.cuda(), q, s, dtype=y), want) and torch.equal(slim.fp8_linear_act(stored(X), q, s, dtype=y), want)


@pytest.mark.parametrize("name", ACTS[1:])
@pytest.mark.parametrize("y", [torch.float32, torch.float16])
def test_activations_over_their_range(slim, name, y):
    """A layer of zeros shows the activation of its bias: small and large values, the tails, what is not finite."""
    z = torch.cat([torch.linspace(-30, 30, 4001), 10.0 ** torch.linspace(-30, 3, 500), -(10.0 ** torch.linspace(-30, 3, 500)), torch.tensor([0.0, -0.0])])
    z = torch.cat([z, torch.tensor([1e30, -1e30, 3e38, -3e38])]) if y == torch.float32 else z
    n = z.numel()
    q, s = slim.fp8_quantize_weights(torch.zeros((n, 8), device="cuda"), transposed=False)
    b = z.to(y)
    for t in (2, 40):
        X = torch.zeros((t, 8), dtype=torch.bfloat16, device="cuda")
        Y = slim.fp8_linear_act(X, q, s, b.cuda(), name, dtype=y)
        want = act(b.double(), name)[0].expand(t, n)
        # (reciprocals and exponentials have no results below 2^-126, the smallest normal number: a factor of that size may be zero, and z times that
        # is missing)
        check(Y, want, torch.nan_to_num(act_steps(b.double(), name) * U * want.abs()) + (1.0 + b.double().abs()) * 2.0 ** -126)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf")], dtype=y).cuda()
    q, s = slim.fp8_quantize_weights(torch.zeros((3, 8), device="cuda"), transposed=False)
    Y = slim.fp8_linear_act(X, q, s, bad, name, dtype=y)
    assert torch.isnan(Y[:, 0]).all() and bool((Y[:, 1] == float("inf")).all())


def neighbours(dz, e, dtype):
    """The 16-bit numbers that dz, off by up to e, may have been rounded to."""
    return (dz - e).to(dtype), (dz + e).to(dtype)


def gradient_range(lo, hi, forms):
    """The least and the greatest that the quantiser makes of numbers between lo and hi: with the scale of either (all of them of a block at
    their nearest to zero, or at their farthest)."""
    far = torch.where(lo.abs() > hi.abs(), lo, hi).double()
    near = torch.where((lo.sign() * hi.sign()) > 0, torch.where(lo.abs() > hi.abs(), hi, lo), torch.zeros_like(lo)).double()
    rows, cols = far.shape
    out = []
    if forms == "cols":
        far, near, lo, hi = far.t(), near.t(), lo.t(), hi.t()
    for scale in (far, near):
        e = ref.quantize(scale)[1]
        s = (2.0 ** e).repeat_interleave(128, 1)[:, :far.shape[1]]
        for v in (lo, hi):
            r = (v.double() / s).clamp(-448.0, 448.0)
            out.append(ref.e4m3(r) * s)
    least, most = torch.stack(out).amin(0), torch.stack(out).amax(0)
    return (least.t(), most.t()) if forms == "cols" else (least, most)


def product_of_range(least, most, B, got, fp32):
    """got against A B for an A between least and most."""
    mid, half = (least + most) / 2, (most - least) / 2
    exact, slack, size = mid @ B, half @ B.abs(), (mid.abs() + half) @ B.abs()
    K = mid.shape[1]
    tol = slack + (2 * K / 8 + 16) * 2.0 ** -23 * size + (0.0 if fp32 else 2.0 ** -10 * size)
    check(got, exact, tol)


def backward(slim, n, m, t, x, dw, name, db):
    W, X, dY = numbers(n, m, torch.float32, 7) * 0.02, numbers(t, m, x, 8), numbers(t, n, x, 9) * 0.01
    Z = (1.5 * torch.randn((t, n), generator=torch.Generator().manual_seed(10))).to(x)
    _, _, qt, st = slim.fp8_quantize_weights(W.cuda())
    dX, dW, dB = slim.fp8_linear_act_backward(dY.cuda(), Z.cuda(), name, X.cuda(), qt, st, dw, db_dtype=db)
    assert dX.dtype == x and dW.dtype == dw and (dB is None) == (db is None)
    slope = act(Z.double(), name)[1]
    dz = dY.double() * slope
    # the slope: 16 half steps of its parts (of a size of up to 1.13), and of the product one more
    e = dY.double().abs() * 24 * U * (slope.abs() + 0.2) if name else torch.zeros_like(dz)
    if name == "relu":
        e = torch.zeros_like(dz)
    lo, hi = neighbours(dz, e, x)
    B = ref.quantize(W, ref.B, ref.B)[2]
    product_of_range(*gradient_range(lo, hi, "rows"), B, dX, False)
    least, most = gradient_range(lo, hi, "cols")
    product_of_range(least.t().contiguous(), most.t().contiguous(), ref.q_cols(X), dW, dw == torch.float32)
    if db is not None:
        # sums of 128 in fp32 (8 one after another, then a tree), then fp64
        check(dB, dz.sum(0), (e + 16 * U * dz.abs()).sum(0))
    return dY, Z, X, qt, st, dX, dW, dB


@pytest.mark.parametrize("n,m", [(1, 1), (5, 3), (127, 129), (300, 1024), (700, 260)])
@pytest.mark.parametrize("t", [1, 17, 128, 301])
@pytest.mark.parametrize("x,dw,db", [(torch.float16, torch.float16, torch.float32), (torch.bfloat16, torch.float32, torch.bfloat16),
                                     (torch.bfloat16, torch.bfloat16, None)])
@pytest.mark.parametrize("name", ["gelu", "silu", None])
def test_backward(slim, n, m, t, x, dw, db, name):
    backward(slim, n, m, t, x, dw, name, db)


@pytest.mark.parametrize("name", ["relu", "gelu_tanh"])
@pytest.mark.parametrize("n,m,t", [(1000, 1501, 301), (2304, 384, 2100)])
def test_backward_of_larger_layers(slim, name, n, m, t):
    """Each gradient alone is the same bytes; strided inputs too."""
    x = torch.bfloat16
    dY, Z, X, qt, st, dX, dW, dB = backward(slim, n, m, t, x, x, name, torch.float32)
    args = dY.cuda(), Z.cuda(), name, X.cuda(), qt, st
    one = slim.fp8_linear_act_backward(*args, dw=False)
    assert torch.equal(one[0], dX) and one[1] is None and one[2] is None
    one = slim.fp8_linear_act_backward(dY.cuda(), Z.cuda(), name, X.cuda(), None, None, dx=False)
    assert torch.equal(one[1], dW) and one[0] is None
    one = slim.fp8_linear_act_backward(dY.cuda(), Z.cuda(), name, None, None, None, dx=False, dw=False, db_dtype=torch.float32)
    assert torch.equal(one[2], dB) and one[0] is None and one[1] is None

    def spread(v, first, gap):
        wide = torch.full((v.shape[0], v.shape[1] + gap), float("nan"), dtype=v.dtype, device="cuda")
        wide[:, first:first + v.shape[1]] = v.cuda()
        return wide[:, first:first + v.shape[1]]

    got = slim.fp8_linear_act_backward(spread(dY, 1, 3), spread(Z, 2, 2), name, spread(X, 3, 7), qt, st, db_dtype=torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(got, (dX, dW, dB)))


def test_without_an_activation_it_is_the_plain_backward_pass(slim):
    for t in (5, 300):
        W, X, dY = numbers(300, 260, torch.float32, 7), numbers(t, 260, torch.bfloat16, 8), numbers(t, 300, torch.bfloat16, 9)
        _, _, qt, st = slim.fp8_quantize_weights(W.cuda())
        want = slim.fp8_linear_backward(dY.cuda(), X.cuda(), qt, st)
        for db in (None, torch.float32):
            got = slim.fp8_linear_act_backward(dY.cuda(), None, None, X.cuda(), qt, st, db_dtype=db)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("n,m,t", [(8192, 2304, 2048), (3576, 4083, 2453), (6462, 2356, 2000), (525, 3810, 5000), (2048, 2304, 5000), (1503, 2000, 97)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_gradients_together_are_those_alone(slim, n, m, t, dtype):
    """The tiles of two products of one launch depend on both; the order of a sum does not."""
    W = (numbers(n, m, torch.float32, 3) * 0.05).cuda()
    X, dY = numbers(t, m, torch.float16, 4).cuda(), numbers(t, n, torch.float16, 5).cuda()
    q, s, qt, st = slim.fp8_quantize_weights(W)
    dX, dW = slim.fp8_linear_backward(dY, X, qt, st, dtype)
    assert torch.equal(dX, slim.fp8_linear_backward(dY, None, qt, st, dw=False)[0])
    assert torch.equal(dW, slim.fp8_linear_backward(dY, X, None, None, dtype, dx=False)[1])
    rows = torch.randperm(t, generator=torch.Generator().manual_seed(1))[:40].cuda()
    A, B = ref.q_rows(dY[rows].cpu()), ref.quantize(W.cpu(), ref.B, ref.B)[2]
    size = A.abs() @ B.abs()
    check(dX[rows], A @ B, ((2 * n / 8 + 16) * 2.0 ** -23 + 2.0 ** -10) * size)


@pytest.mark.parametrize("name", ACTS[1:])
def test_slopes_are_differences_of_the_activations(slim, name):
    """The bias gradient of one token is the slope itself; differences of the formula in 64 bits."""
    z = torch.linspace(-9, 9, 1800).half()
    z = z[z != 0]
    n = z.numel()
    one = torch.ones((1, n), dtype=torch.float16, device="cuda")
    db = slim.fp8_linear_act_backward(one, z.cuda().view(1, n), name, None, None, None, dx=False, dw=False, db_dtype=torch.float32)[2]
    h = 1e-4 if name != "relu" else 1e-8
    diff = (act(z.double() + h, name)[0] - act(z.double() - h, name)[0]) / (2 * h)
    # central differences: h^2 / 6 of a third derivative below 10, rounding 1e-15 / h (9e-8 for relu's h); the kernel 24 half steps
    assert float((db.double().cpu() - diff).abs().max()) <= 1e-8 * 10 / 6 + 1e-14 / h + 24 * U * 1.2


def test_special_values(slim):
    """What is not finite in a token's gradient or kept values stays in its rows of dX; large values have slopes of zero and one."""
    n, m, t = 200, 130, 60
    W, X, dY = numbers(n, m, torch.float32, 7), numbers(t, m, torch.bfloat16, 8), numbers(t, n, torch.bfloat16, 9)
    Z = numbers(t, n, torch.bfloat16, 11)
    _, _, qt, st = slim.fp8_quantize_weights(W.cuda())
    for name in ACTS[1:]:
        clean = slim.fp8_linear_act_backward(dY.cuda(), Z.cuda(), name, None, qt, st, dw=False)[0]
        z, dy = Z.clone(), dY.clone()
        z[3, 5], dy[7, 9] = float("nan"), float("inf")
        z[7, 9] = 1.0
        dx = slim.fp8_linear_act_backward(dy.cuda(), z.cuda(), name, None, qt, st, dw=False)[0]
        keep = [i for i in range(t) if i not in (3, 7)]
        assert torch.isnan(dx[3]).all() and torch.isnan(dx[7]).all() and torch.equal(dx[keep], clean[keep])
        big = torch.tensor([[1e4, -1e4, 3e38, -3e38]]).bfloat16()
        db = slim.fp8_linear_act_backward(torch.ones_like(big).cuda(), big.cuda(), name, None, None, None, dx=False, dw=False, db_dtype=torch.float32)[2]
        assert db.tolist() == [1.0, 0.0, 1.0, 0.0], (name, db)


def test_no_tokens_and_rows_behind_the_last(slim):
    from paper_2405_14917_amd import binding as B
    import ctypes
    W = numbers(300, 200, torch.float32, 1).cuda()
    q, s, qt, st = slim.fp8_quantize_weights(W)
    none = torch.empty((0, 200), dtype=torch.bfloat16, device="cuda")
    Y, Z = slim.fp8_linear_act(none, q, s, act="silu", keep=True)
    assert Y.shape == Z.shape == (0, 300)
    dX, dW, db = slim.fp8_linear_act_backward(Y, Z, "silu", none, qt, st, db_dtype=torch.float32)
    assert dX.shape == (0, 200) and not dW.any() and not db.any()
    for t in (3, 150):
        X = numbers(t, 200, torch.bfloat16, 2).cuda()
        Y, Z = (torch.full((t + 1, 310), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        e = B.SlimEpilogue(None, B.F32, 2, None, 0, Z.data_ptr(), 310)
        assert slim.lib.slim_fp8_linear_act(slim.ctx, X.data_ptr(), B.BF16, t, 200, None, 0, None, 0, q.data_ptr(), q.stride(0), s.data_ptr(), s.stride(0), 300,
                                            200, ctypes.byref(e), Y.data_ptr(), B.BF16, 310) == B.SLIM_OK
        want = slim.fp8_linear_act(X, q, s, act="gelu", keep=True)
        for got, w in zip((Y, Z), want):
            assert torch.equal(got[:t, :300], w) and bool((got[t] == 7).all()) and bool((got[:, 300:] == 7).all())


@pytest.mark.parametrize("n,m,t", [(1000, 1504, 301), (4096, 1030, 90), (520, 9000, 96)])
def test_a_workspace_of_the_queried_size_is_enough(n, m, t):
    from paper_2405_14917_amd import binding
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    base = binding.Slim("cuda:0")
    q, s, qt, st = base.fp8_quantize_weights(numbers(n, m, torch.float32, 1).cuda())
    X, dY, Z = numbers(t, m, torch.bfloat16, 2).cuda(), numbers(t, n, torch.bfloat16, 3).cuda(), numbers(t, n, torch.bfloat16, 4).cuda()
    want = base.fp8_linear_act(X, q, s, act="gelu"), base.fp8_linear_act_backward(dY, Z, "gelu", X, qt, st, db_dtype=torch.float32)
    for need, call, i in ((binding.fp8_linear_act_workspace(n, m, t, False, torch.bfloat16, ncu), lambda c: (c.fp8_linear_act(X, q, s, act="gelu"),), 0),
                          (binding.fp8_linear_act_backward_workspace(n, m, t, num_cus=ncu),
                           lambda c: c.fp8_linear_act_backward(dY, Z, "gelu", X, qt, st, db_dtype=torch.float32), 1)):
        for size, ok in ((need, True), (need - 256, False)):
            if size <= 0:
                continue
            c = binding.Slim("cuda:0", workspace_bytes=size)
            try:
                if ok:
                    got = call(c)
                    assert all(torch.equal(a, b) for a, b in zip(got, want[i] if i else (want[0],)))
                else:
                    with pytest.raises(binding.SlimError) as e:
                        call(c)
                    assert e.value.status == binding.ERR_ALLOC
                torch.cuda.synchronize()
            finally:
                c.close()
    base.close()


def test_refusals(slim):
    from paper_2405_14917_amd import binding
    W, X = numbers(130, 200, torch.float32, 1).cuda(), numbers(5, 200, torch.bfloat16, 2).cuda()
    q, s, qt, st = slim.fp8_quantize_weights(W)
    xq, xs = stored(X.cpu())
    Y, Z = slim.fp8_linear_act(X, q, s, act="silu", keep=True)
    b = torch.zeros(130, device="cuda")
    for bad in (lambda: slim.fp8_linear_act(X[:, :199], q, s), lambda: slim.fp8_linear_act(X, q, s, b[:129]), lambda: slim.fp8_linear_act(X, q, s, act="tanh"),
                lambda: slim.fp8_linear_act(X, q, s, residual=Y.float(), dtype=torch.bfloat16), lambda: slim.fp8_linear_act(X, q, s, residual=Y[:4]),
                lambda: slim.fp8_linear_act((xq, xs[:4]), q, s), lambda: slim.fp8_linear_act((xq.view(torch.uint8), xs), q, s),
                lambda: slim.fp8_linear_act((xq[:, :100], xs), q, s), lambda: slim.fp8_linear_act(X.cpu(), q, s),
                lambda: slim.fp8_linear_act_backward(Y, None, "silu", X, qt, st), lambda: slim.fp8_linear_act_backward(Y, Z[:4], "silu", X, qt, st),
                lambda: slim.fp8_linear_act_backward(Y, Z.float(), "silu", X, qt, st), lambda: slim.fp8_linear_act_backward(Y, Z, "silu", X[:4], qt, st),
                lambda: slim.fp8_linear_act_backward(Y, Z, "silu", X, None, None), lambda: slim.fp8_linear_act_backward(Y, Z, "silu", None, None, None, dx=False, dw=False)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: slim.fp8_linear_act(X.float(), q, s), lambda: slim.fp8_linear_act(X, q, s, dtype=torch.float64),
                lambda: slim.fp8_linear_act(X, q, s, b.half()), lambda: slim.fp8_linear_act_backward(Y, Z, "silu", X, qt, st, db_dtype=torch.float64)):
        with pytest.raises(binding.SlimError) as e:
            bad()
        assert e.value.status == binding.ERR_UNSUPPORTED

"""The 8-bit linear layer where it takes a launch that quantises and one that multiplies (fp8_rows, fp8_tiles, fp8_gemm): every test asserts that
its sizes are not those of the one-launch kernel.

Tolerances as in test_gpu_fp8_linear.  Small integers have none: they are e4m3 numbers, their products and all partial sums are integers far below
2^13 in a group of eight and below 2^24 in all, so the sums are exact on either matrix cores and the result is the integer, rounded once."""
import pytest
import torch

import fp8_reference as ref
from test_gpu_fp8_linear import close, numbers, slim  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def two_launches(n, m, t, y):
    from paper_2405_14917_amd import binding
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    assert binding.fp8_linear_workspace(n, m, t, y, ncu) > 0


def spoil_scale_padding(s):
    """What pads a row of scales is not used."""
    torch.as_strided(s, (s.shape[0], s.stride(0)), (s.stride(0), 1))[:, s.shape[1]:] = 255


def spread(v, first, gap):
    """The same matrix with rows that start anywhere, NaN between them."""
    wide = torch.full((v.shape[0] + 1, v.shape[1] + gap), float("nan"), dtype=v.dtype, device="cuda")
    wide[:-1, first:first + v.shape[1]] = v.cuda()
    return wide[:-1, first:first + v.shape[1]]


def integers(rows, cols, seed, largest=3):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-largest, largest + 1, (rows, cols), generator=g).float()


def by_blocks(cols, sign):
    """Powers of two that differ from block to block of 128."""
    return 2.0 ** (sign * (torch.arange(cols) // 128 % 3).float())


def exact_product(A, B):
    return A.double().cuda() @ B.double().cuda().t()


@pytest.mark.parametrize("x", [F16, BF16])
@pytest.mark.parametrize("wide_out", [False, True])
def test_activations_are_quantised_as_defined(slim, x, wide_out):  # noqa: F811
    """A layer that hands its inputs through shows Q(X) itself: every value there is, the borders of a scale among them."""
    t, m, y = 6000, 384, F32 if wide_out else x
    two_launches(m, m, t, y)
    X = (torch.arange(t * m, dtype=torch.int32) * 7919 % 65536).to(torch.uint16).view(x).reshape(t, m).clone()
    X[~torch.isfinite(X)] = 1.5
    if x == BF16:
        X = (X.double().sign() * X.double().abs().clamp(2.0 ** -100, 2.0 ** 100)).to(x)     # exact through the identity
    X[0, :128], X[1, :128], X[2, :128] = 448.0, 449.0, 0.0
    X[3, :128] = torch.linspace(0, 448, 128).to(x)
    q, s = slim.fp8_quantize_weights(torch.eye(m).cuda(), transposed=False)
    Y = slim.fp8_linear(X.cuda(), q, s, y)
    # (a stored number times its scale is one of X's type, but for the largest of fp16, which becomes 65536)
    assert torch.equal(Y.cpu(), ref.q_rows(X).to(y))


@pytest.mark.parametrize("y", [BF16, F32])
def test_what_is_not_finite_stays_in_its_token(slim, y):  # noqa: F811
    n, m, t = 640, 700, 3000
    two_launches(n, m, t, y)
    X = numbers(t, m, BF16, 2)
    X[t - 1, 7] = X[t - 1, 690] = X[5, 300] = 0.0                # (the blocks' scales stay what they are)
    q, s = slim.fp8_quantize_weights(numbers(n, m, F32, 1).cuda(), transposed=False)
    spoil_scale_padding(s)
    clean = slim.fp8_linear(X.cuda(), q, s, y)
    X[t - 1, 7], X[t - 1, 690], X[5, 300] = float("inf"), float("nan"), -float("inf")
    Y = slim.fp8_linear(X.cuda(), q, s, y)
    keep = torch.ones(t, dtype=torch.bool)
    keep[[5, t - 1]] = False
    assert torch.isnan(Y[~keep]).all() and torch.equal(Y[keep], clean[keep]) and torch.isfinite(clean).all()


def test_what_is_not_finite_stays_in_its_gradients(slim):  # noqa: F811
    """dY[i, j]: in row i of dX and row j of dW; X[i, k]: in column k of dW."""
    n, m, t = 150, 333, 300
    X, dY = numbers(t, m, F16, 3), numbers(t, n, F16, 4)
    dY[7, 140] = dY[299, 3] = X[200, 332] = X[5, 0] = 0.0
    _, _, qt, st = slim.fp8_quantize_weights(numbers(n, m, F32, 5).cuda())
    spoil_scale_padding(st)
    gx, gw = slim.fp8_linear_backward(dY.cuda(), X.cuda(), qt, st)
    dY[7, 140], dY[299, 3], X[200, 332], X[5, 0] = float("inf"), float("nan"), float("nan"), -float("inf")
    dX, dW = slim.fp8_linear_backward(dY.cuda(), X.cuda(), qt, st)
    kx, kn, km = torch.ones(t, dtype=torch.bool), torch.ones(n, dtype=torch.bool), torch.ones(m, dtype=torch.bool)
    kx[[7, 299]] = kn[[140, 3]] = km[[332, 0]] = False
    assert torch.isnan(dX[~kx]).all() and torch.equal(dX[kx], gx[kx])
    assert torch.isnan(dW[~kn]).all() and torch.isnan(dW[:, ~km]).all() and torch.equal(dW[kn][:, km], gw[kn][:, km])
    assert torch.isfinite(gx).all() and torch.isfinite(gw).all()


# tiles of 64, 128 and 256 rows, each whole and in parts along the contraction, at either type of output
SHAPES = [(520, 700, 1500), (520, 3000, 300), (1000, 700, 2050), (300, 9000, 1500), (520, 6000, 1000), (4100, 3000, 2050), (1000, 16000, 4100),
          (1000, 12000, 2050), (300, 20001, 300)]


@pytest.mark.parametrize("n,m,t", SHAPES)
@pytest.mark.parametrize("x,y", [(F16, F16), (BF16, BF16), (F16, F32)])
def test_integers_are_exact(slim, n, m, t, x, y):  # noqa: F811
    two_launches(n, m, t, y)
    X, W = integers(t, m, 1) * by_blocks(m, 1), integers(n, m, 2) * by_blocks(m, -1)
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    spoil_scale_padding(s)
    assert torch.equal(slim.fp8_linear(X.to(x).cuda(), q, s, y), exact_product(X, W).to(y))


@pytest.mark.parametrize("n,m,t", [(300, 200, 5000), (1090, 2200, 260), (2100, 1100, 1025), (900, 700, 9000), (4100, 3000, 2100), (257, 129, 17)])
@pytest.mark.parametrize("x,dw", [(F16, F16), (BF16, F32), (BF16, BF16)])
def test_integer_gradients_are_exact(slim, n, m, t, x, dw):  # noqa: F811
    X, W, dY = integers(t, m, 3), integers(n, m, 4), integers(t, n, 5)
    dY[t // 2] = 0.0
    _, _, qt, st = slim.fp8_quantize_weights(W.cuda())
    spoil_scale_padding(st)
    dX, dW = slim.fp8_linear_backward(dY.to(x).cuda(), X.to(x).cuda(), qt, st, dw)
    assert torch.equal(dX, exact_product(dY, W.t()).to(x)) and torch.equal(dW, exact_product(dY.t(), X.t()).to(dw))


@pytest.mark.parametrize("n,m,t", [(520, 701, 1500), (4100, 3000, 2050)])
@pytest.mark.parametrize("x,y", [(F16, F16), (BF16, BF16), (F16, F32)])
def test_forward(slim, n, m, t, x, y):  # noqa: F811
    two_launches(n, m, t, y)
    W, X = numbers(n, m, F32, 3) * 0.02, numbers(t, m, x, 4)
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    Y = slim.fp8_linear(X.cuda(), q, s, y)
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    close(Y, exact_product(A, B).cpu(), exact_product(A.abs(), B.abs()).cpu(), m, False)


@pytest.mark.parametrize("y", [F16, F32])
def test_strides_and_alignment(slim, y):  # noqa: F811
    from paper_2405_14917_amd import binding as b
    n, m, t = 641, 701, 3000
    two_launches(n, m, t, y)
    X = numbers(t, m, F16, 14)
    q, s = slim.fp8_quantize_weights((numbers(n, m, F32, 13) * 0.02).cuda(), transposed=False)
    base = slim.fp8_linear(X.cuda(), q, s, y)
    for first, gap in ((0, 1), (1, 2), (3, 6), (5, 8)):
        assert torch.equal(slim.fp8_linear(spread(X, first, gap), q, s, y), base)
    # outputs in a wider matrix, through the C entry point
    Y, Xc = torch.full((t, n + 5), 7.0, dtype=y, device="cuda"), X.cuda()
    assert slim.lib.slim_fp8_linear(slim.ctx, Xc.data_ptr(), b.F16, t, m, q.data_ptr(), q.stride(0), s.data_ptr(), s.stride(0), n, m,
                                    Y.data_ptr() + Y.element_size(), b.F16 if y == F16 else b.F32, n + 5) == b.SLIM_OK
    assert torch.equal(Y[:, 1:n + 1], base) and bool((Y[:, 0] == 7).all()) and bool((Y[:, n + 1:] == 7).all())


@pytest.mark.parametrize("n,m", [(16, 128), (127, 129), (130, 511), (300, 1024), (700, 260)])
@pytest.mark.parametrize("t", [17, 33, 130])
def test_the_one_launch_kernel_keeps_24_bits(slim, n, m, t):  # noqa: F811
    """Sizes of more than 16 tokens that it takes: its sums have the tolerance of fp32 ones at 16-bit outputs too."""
    from paper_2405_14917_amd import binding
    assert binding.fp8_linear_workspace(n, m, t, F16, torch.cuda.get_device_properties(0).multi_processor_count) == 0
    W, X = numbers(n, m, F32, 3) * 0.02, numbers(t, m, F16, 4)
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    close(slim.fp8_linear(X.cuda(), q, s), A @ B.t(), A.abs() @ B.abs().t(), m, True)


@pytest.mark.parametrize("n,m,t", [(520, 700, 1500), (300, 9000, 1500), (1000, 700, 2050), (4100, 3000, 2050)])
@pytest.mark.parametrize("x", [F16, BF16])
def test_what_the_e4m3_cores_drop(slim, n, m, t, x):  # noqa: F811
    """Of eight products each loses less than 2^-13 of the largest P, without a bias: in squares 8 2^-26 / 3 P^2 a group, P^2 at most the sum of its
    eight squares, so in all 8 / 3 2^-26 of the norm of the result, beside its rounding.  (Normal data: a result's norm is that of its products.)"""
    two_launches(n, m, t, x)
    g = torch.Generator().manual_seed(n)
    X, W = torch.randn((t, m), generator=g).to(x), torch.randn((n, m), generator=g)
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    Y = slim.fp8_linear(X.cuda(), q, s).double()
    exact = exact_product(ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2])
    off, rounding = float((Y - exact).norm() / exact.norm()), float((exact.to(x).double() - exact).norm() / exact.norm())
    assert off ** 2 - rounding ** 2 <= 8 / 3 * 2.0 ** -26, (off, rounding)

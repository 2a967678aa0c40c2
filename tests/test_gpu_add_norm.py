"""The norm of the residual stream, forward and backward, against its formulas in 64 bits.

The sum h is one rounding of a sum of two numbers: exact here, since both sides take it in fp32.  From h on the tolerances are those of the norms
(test_gpu_norm.py); the 8-bit form is, number for number, what the quantiser's definition (fp8_reference.py) makes of the rounded output; the
gradient that reaches the stream past the norm adds one rounding."""
import pytest
import torch

import fp8_reference as ref
from test_gpu_norm import HALF, TINY, TYPES, U, close, data, statistics

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


def cuda(*v):
    return [None if t is None else t.cuda() for t in v]


def problem(rows, cols, x, w, seed):
    X, dY, wt, b = data(rows, cols, x, w, seed)
    R, dH, _, _ = data(rows, cols, x, w, seed + 1000)
    return X, R, dY, dH, wt, b


def check_stored(o, Y):
    """q and s are what the quantiser makes of Y; a row is padded with zeros to its last block."""
    rows, cols = Y.shape
    num, e, _ = ref.quantize(Y.cpu())
    same = lambda a, b: torch.equal(torch.nan_to_num(a, nan=1e9), torch.nan_to_num(b, nan=1e9))
    assert o.q.shape == Y.shape and same(o.q.cpu().double(), num) and torch.equal(o.s.cpu().double() - 127, e)
    assert o.q.stride(0) % 128 == 0 and o.s.stride(0) % 4 == 0
    padded = -(-cols // 128) * 128
    assert not torch.as_strided(o.q, (rows, padded), (o.q.stride(0), 1)).view(torch.uint8)[:, cols:].any()


def check(slim, X, R, dY, dH, w, b, eps, rms, given=None):
    Xg, Rg, dYg, dHg, wg, bg = given or cuda(X, R, dY, dH, w, b)
    o = slim.add_norm(Xg, Rg, wg, bg, eps, rms=rms, e4m3=True, stats=True)
    H = X if R is None else (X.float() + R.float()).to(X.dtype)
    assert torch.equal(o.H.cpu(), H) and (o.mean is None) == rms
    m, d, r, e_d, e_r, c = statistics(H, eps, rms)
    wd, xh = w.double(), d * r
    e_x = e_d * r + xh.abs() * (e_r + 2 * U)
    close(o.Y, xh * wd + (0.0 if b is None else b.double()), e_x * wd.abs() + U * (xh * wd).abs(), X.dtype)
    check_stored(o, o.Y)
    only = slim.add_norm(Xg, Rg, wg, bg, eps, rms=rms, y=False, e4m3=True)
    bare = slim.add_norm(Xg, Rg, wg, bg, eps, rms=rms)
    assert only.Y is None and bare.q is None and bare.mean is None and torch.equal(bare.Y, o.Y)
    assert torch.equal(only.q.view(torch.uint8), o.q.view(torch.uint8)) and torch.equal(only.s, o.s) and torch.equal(only.H, o.H)
    dX, dw, db = slim.add_norm_backward(dYg, dHg, o.H, wg, o.mean, o.rstd, bias=b is not None)
    g = dY.double() * wd
    mg, mgx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    if rms:
        mg = torch.zeros_like(mg)
    e_mgx = c * U * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * e_x).mean(1, keepdim=True) + 2 * U * (g * xh).abs().mean(1, keepdim=True)
    e_mg = (c + 2) * U * g.abs().mean(1, keepdim=True)
    t = g - mg - xh * mgx
    e_t = 4 * U * (g.abs() + mg.abs() + (xh * mgx).abs()) + e_mg + e_x * mgx.abs() + xh.abs() * e_mgx + e_x * e_mgx
    past = torch.zeros_like(t) if dH is None else dH.double()
    close(dX, t * r + past, r * e_t + (e_r + 2 * U) * (t * r).abs() + U * ((t * r).abs() + past.abs()), X.dtype)
    rows = X.shape[0]
    k = rows / 1024 + 1024 / 8 + 16
    close(dw, (dY.double() * xh).sum(0), k * U * (dY.double() * xh).abs().sum(0) + (dY.double().abs() * e_x).sum(0), w.dtype)
    if b is not None:
        close(db, dY.double().sum(0), k * U * dY.double().abs().sum(0), w.dtype)
    else:
        assert db is None
    return o, dX, dw, db


@pytest.mark.parametrize("cols", [1, 7, 64, 100, 127, 129, 513, 1501, 2048, 4096, 6001, 8192, 12288, 16384])
@pytest.mark.parametrize("x,w", TYPES)
@pytest.mark.parametrize("rms,bias", [(False, True), (True, False)])
def test_every_width(slim, cols, x, w, rms, bias):
    X, R, dY, dH, wt, b = problem(21, cols, x, w, cols)
    check(slim, X, R, dY, dH, wt, b if bias else None, 1e-5, rms)


@pytest.mark.parametrize("rows", [1, 2, 5, 17, 65, 1030, 5000])
@pytest.mark.parametrize("cols", [96, 1000, 1500])
@pytest.mark.parametrize("rms,bias,stream", [(False, False, True), (True, True, True), (True, False, False)])
def test_every_height(slim, rows, cols, rms, bias, stream):
    """Also without a stream to add, and without a gradient past the norm."""
    X, R, dY, dH, wt, b = problem(rows, cols, torch.bfloat16, torch.float32, rows)
    check(slim, X, R if stream else None, dY, dH if stream else None, wt, b if bias else None, 1e-6, rms)


@pytest.mark.parametrize("x,cols", [(torch.float32, 16385), (torch.bfloat16, 32769), (torch.float16, 70001)])
@pytest.mark.parametrize("rms", [False, True])
def test_rows_longer_than_registers_hold(slim, x, cols, rms):
    X, R, dY, dH, wt, b = problem(3, cols, x, torch.float32, 3)
    check(slim, X, R, dY, dH, wt, b, 1e-5, rms)


@pytest.mark.parametrize("x", [torch.float32, torch.bfloat16])
def test_the_8_bit_form_feeds_the_linear_layer(slim, x):
    """The layer gives the same bytes for the 8-bit form as for the 16-bit outputs that it quantises itself."""
    for rows, cols, n in ((1, 300, 130), (16, 1024, 700), (40, 512, 96), (300, 1100, 1500)):
        X, R, _, _, wt, b = problem(rows, cols, x, torch.float32, rows)
        W = torch.randn((n, cols), generator=torch.Generator().manual_seed(1)) * 0.05
        q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
        o = slim.add_norm(*cuda(X, R, wt, b), e4m3=True)
        for y in (torch.bfloat16, torch.float32):
            got = slim.fp8_linear_act((o.q, o.s), q, s, dtype=y)
            if x != torch.float32:
                assert torch.equal(got, slim.fp8_linear(o.Y, q, s, y))
            else:
                want = ref.q_rows(o.Y.cpu()) @ ref.quantize(W, ref.B, ref.B)[2].t()
                assert float((got.double().cpu() - want).norm() / want.norm()) < (1e-2 if y == torch.bfloat16 else 1e-5)


def test_special_rows(slim):
    """What is not finite stays in its row and becomes NaN in 8 bits; rows of one value, of zeros."""
    X, R, dY, dH, wt, b = problem(8, 300, torch.bfloat16, torch.float32, 7)
    X[1], R[1] = 3.0, -3.0
    X[2], R[2] = 2.0, 1.0
    clean, _, _, _ = check(slim, X, R, dY, dH, wt, b, 1e-5, False)
    assert not clean.H[1].any() and torch.equal(clean.Y[1].cpu(), b.to(torch.bfloat16)) and torch.equal(clean.Y[2].cpu(), b.to(torch.bfloat16))
    X[3, 5], R[4, 299], X[6, 0], R[6, 0] = float("nan"), float("inf"), float("inf"), -float("inf")
    for rms in (False, True):
        ok = slim.add_norm(*cuda(torch.nan_to_num(X, posinf=1.0), torch.nan_to_num(R, posinf=1.0, neginf=1.0), wt, b), rms=rms, e4m3=True)
        o = slim.add_norm(*cuda(X, R, wt, b), rms=rms, e4m3=True)
        check_stored(o, o.Y)
        assert torch.isnan(o.Y[3]).all() and torch.isnan(o.Y[6]).all() and torch.isnan(o.Y[4]).any()
        for k in (0, 1, 2, 5, 7):
            assert torch.equal(o.Y[k], ok.Y[k]) and torch.equal(o.q[k].view(torch.uint8), ok.q[k].view(torch.uint8)) and torch.equal(o.s[k], ok.s[k])
    big = torch.full((2, 200), 60000.0, dtype=torch.float16)                 # the sum leaves fp16
    o = slim.add_norm(*cuda(big, big, torch.ones(200), None), e4m3=True)
    assert torch.isinf(o.H).all() and torch.isnan(o.Y).all() and torch.isnan(o.q.float()).all() and bool((o.s == 1).all())


@pytest.mark.parametrize("x", [torch.float32, torch.float16])
def test_strides_and_alignment(slim, x):
    rows, cols = 70, 301
    X, R, dY, dH, wt, b = problem(rows, cols, x, x, 8)
    base = check(slim, X, R, dY, dH, wt, b, 1e-5, False)

    def spread(v, first, gap):
        wide = torch.full((rows, cols + gap), float("nan"), dtype=x, device="cuda")
        wide[:, first:first + cols] = v.cuda()
        return wide[:, first:first + cols]

    off = torch.full((cols + 1,), float("nan"), dtype=x, device="cuda")
    off[1:] = wt.cuda()
    for first, gap in ((1, 1), (3, 7), (0, 2)):
        got = check(slim, X, R, dY, dH, wt, b, 1e-5, False,
                    (spread(X, first, gap), spread(R, gap - first, gap), spread(dY, 0, gap), spread(dH, first, gap + 4), off[1:], b.cuda()))
        for p, q in zip(got[1:] + (got[0].Y, got[0].H), base[1:] + (base[0].Y, base[0].H)):
            assert torch.equal(p, q)


@pytest.mark.parametrize("cols,x", [(300, torch.bfloat16), (4096, torch.float16), (9000, torch.float32), (33000, torch.bfloat16), (17000, torch.float32)])
def test_the_stream_may_stay_in_its_place(slim, cols, x):
    """H over R or over X; dX over dH, dY or H (C interface)."""
    from paper_2405_14917_amd import binding as B
    X, R, dY, dH, wt, b = problem(40, cols, x, torch.float32, cols)
    Xg, Rg, dYg, dHg, wg, bg = cuda(X, R, dY, dH, wt, b)
    o = slim.add_norm(Xg, Rg, wg, bg, e4m3=True, stats=True)
    for which in (0, 1):
        v = [Xg.clone(), Rg.clone()]
        p = slim.add_norm(*v, wg, bg, e4m3=True, H=v[which])
        assert p.H is v[which] and torch.equal(p.H, o.H) and torch.equal(p.Y, o.Y) and torch.equal(p.s, o.s)
        assert torch.equal(p.q.view(torch.uint8), o.q.view(torch.uint8))
    dX, dw, db = slim.add_norm_backward(dYg, dHg, o.H, wg, o.mean, o.rstd, bias=True)
    ptr = lambda t: t.data_ptr()
    for over in range(3):
        v = [dYg.clone(), dHg.clone(), o.H.clone()]
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        assert slim.lib.slim_add_norm_backward(slim.ctx, *map(ptr, v), B._DT[x], 40, cols, cols, cols, cols, ptr(wg), B.F32, ptr(o.mean), ptr(o.rstd),
                                               ptr(v[over]), cols, ptr(dw2), ptr(db2)) == B.SLIM_OK
        assert torch.equal(v[over], dX) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_rows_behind_the_last_one_are_left_alone(slim):
    from paper_2405_14917_amd import binding as B
    X, R, _, _, wt, _ = problem(6, 130, torch.bfloat16, torch.float32, 5)
    Xg, Rg, wg = cuda(X, R, wt)
    H, Y = (torch.full((6, 150), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, s = torch.full((6, 384), 9, dtype=torch.uint8, device="cuda"), torch.full((6, 4), 9, dtype=torch.uint8, device="cuda")
    p = lambda t: t.data_ptr()
    assert slim.lib.slim_add_norm(slim.ctx, p(Xg), p(Rg), B.BF16, 5, 130, 130, 130, p(wg), None, B.F32, 1e-5, 1, p(H), 150, p(Y), 150, p(q), 384, p(s), 4,
                                  None, None) == B.SLIM_OK
    assert bool((H[5] == 7).all()) and bool((Y[5] == 7).all()) and bool((H[:, 130:] == 7).all()) and bool((Y[:, 130:] == 7).all())
    assert bool((q[5] == 9).all()) and bool((q[:, 256:] == 9).all()) and not q[:5, 130:256].any() and bool((s[5] == 9).all()) and bool((s[:, 2:] == 9).all())


def test_gradients_are_differences_of_the_outputs(slim):
    """Of the formula in 64 bits, at the sum in fp32 (which rounds nothing of these numbers)."""
    X, R, dY, dH, wt, b = problem(4, 50, torch.float32, torch.float32, 6)
    X, R = ((v * 2 ** 10).round() / 2 ** 10 for v in (X, R))

    def f(x, rms):
        d = x - (0.0 if rms else x.mean(1, keepdim=True))
        return ((d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * wt.double() + b.double()) * dY.double()).sum() + (x * dH.double()).sum()

    for rms in (False, True):
        o, dX, _, _ = check(slim, X, R, dY, dH, wt, b, 1e-5, rms)
        h = 1e-5
        for i, j in ((0, 0), (3, 49), (2, 17)):
            up, down = X.double() + R.double(), X.double() + R.double()
            up[i, j] += h
            down[i, j] -= h
            diff = float(f(up, rms) - f(down, rms)) / (2 * h)
            # central differences: h^2 / 6 of the third derivative (below 1e3 here) and the sums' 1e-15 over h
            assert abs(float(dX[i, j]) - diff) <= 1e-7 + 1e-5 * max(1.0, abs(diff))


def test_no_rows(slim):
    w = torch.ones(33, device="cuda")
    X = torch.empty((0, 33), device="cuda")
    o = slim.add_norm(X, X, w, w, e4m3=True, stats=True)
    dX, dw, db = slim.add_norm_backward(X, X, X, w, o.mean, o.rstd, bias=True)
    assert o.Y.shape == o.H.shape == dX.shape == (0, 33) and o.q.shape == (0, 33) and not dw.any() and not db.any()


def test_a_workspace_of_the_queried_size_is_enough():
    from paper_2405_14917_amd import binding
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    X, R, dY, dH, w, _ = cuda(*problem(2000, 999, torch.float32, torch.float32, 10))
    need = binding.layer_norm_backward_workspace(2000, 999, True, torch.float32, ncu)
    for size, ok in ((need, True), (need - 256, False)):
        s = binding.Slim("cuda:0", workspace_bytes=size)
        try:
            o = s.add_norm(X, R, w, stats=True)
            if ok:
                s.add_norm_backward(dY, dH, o.H, w, o.mean, o.rstd, bias=True)
            else:
                with pytest.raises(binding.SlimError) as e:
                    s.add_norm_backward(dY, dH, o.H, w, o.mean, o.rstd, bias=True)
                assert e.value.status == binding.ERR_ALLOC
            torch.cuda.synchronize()
        finally:
            s.close()


def test_refusals(slim):
    from paper_2405_14917_amd import binding
    X, R, dY, dH, w, b = cuda(*problem(4, 32, torch.float32, torch.float32, 11))
    o = slim.add_norm(X, R, w, stats=True)
    for bad in (lambda: slim.add_norm(X, R[:3], w), lambda: slim.add_norm(X, R.half(), w), lambda: slim.add_norm(X, R, w, y=False),
                lambda: slim.add_norm(X, R.cpu(), w), lambda: slim.add_norm(X, R, w, H=X[:2]), lambda: slim.add_norm(X, None, w, H=R),
                lambda: slim.add_norm(X, R, w[:31]), lambda: slim.add_norm(X.t(), R.t(), w[:4]),
                lambda: slim.add_norm_backward(dY, dH[:3], o.H, w, o.mean, o.rstd), lambda: slim.add_norm_backward(dY.half(), dH, o.H, w, o.mean, o.rstd),
                lambda: slim.add_norm_backward(dY, dH, o.H, w, o.mean.double(), o.rstd)):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: slim.add_norm(X.double(), R.double(), w.double()), binding.ERR_UNSUPPORTED),
                        (lambda: slim.add_norm(X, R, w, eps=-1.0), binding.ERR_INVALID_ARG)):
        with pytest.raises(binding.SlimError) as e:
            bad()
        assert e.value.status == status

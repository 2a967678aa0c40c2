"""Layer norm and its form without the mean, forward and backward, against their formulas in 64 bits.

Tolerances (u = 2^-24, half a step of fp32; n columns).  Sums of n terms in fp32, a lane's one after another and then by a tree, are off by at
most (n / 64 + 16) u of the sum of magnitudes for rows of up to 16384 columns, n / 1024 + 16 beyond (the lanes of 16 wavefronts); call it
c u.  So the mean is off by c u mean|x|; the deviations by that and two roundings; r and xh by the variance's relative error 2 (c + 4) u / 2
and a few roundings: each gradient by sums of what it is made of.  Then half a step of the output's type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -140}


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


def data(rows, cols, x, w, seed, offset=0.3):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    X = (r(rows, cols) * torch.exp(r(rows, 1)) + offset * r(1, cols)).to(x)
    dY = (r(rows, cols) * torch.exp(0.5 * r(rows, 1))).to(x)
    return X, dY, (1 + 0.3 * r(cols)).to(w), (0.1 * r(cols)).to(w)


def close(got, want, tol, dtype):
    got = got.double().cpu()
    tol = tol + HALF[dtype] * (want.abs() + tol) + TINY[dtype]
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs() / tol).max()))


def statistics(X, eps, rms):
    x = X.double()
    mean = torch.zeros(x.shape[0], 1, dtype=torch.float64) if rms else x.mean(1, keepdim=True)
    d = x - mean
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    n = x.shape[1]
    c = (n / 64 if n <= 16384 else n / 1024) + 16
    e_d = 0.0 if rms else c * U * x.abs().mean(1, keepdim=True)                 # of a deviation
    e_d = e_d + 2 * U * (x.abs() + mean.abs())
    # v + eps = 1 / r^2: the sum's own roundings, and those of the deviations
    e_v = (c + 4) * U + 2 * (e_d * d.abs()).mean(1, keepdim=True) * r * r
    e_r = e_v / 2 + 4 * U                                                        # relative, of r
    return mean, d, r, e_d, e_r, c


def check(slim, X, dY, w, b, eps, rms, given=None):
    rows, cols = X.shape
    Xg, dYg, wg, bg = given or (X.cuda(), dY.cuda(), w.cuda(), None if b is None else b.cuda())
    Y, mean, rstd = slim.layer_norm(Xg, wg, bg, eps, rms=rms, stats=True)
    assert torch.equal(Y, slim.layer_norm(Xg, wg, bg, eps, rms=rms)) and (mean is None) == rms
    dX, dw, db = slim.layer_norm_backward(dYg, Xg, wg, mean, rstd, bias=b is not None)
    m, d, r, e_d, e_r, c = statistics(X, eps, rms)
    wd, xh = w.double(), d * r
    e_x = e_d * r + xh.abs() * (e_r + 2 * U)
    want = xh * wd + (0.0 if b is None else b.double())
    close(Y, want, e_x * wd.abs() + U * (xh * wd).abs(), X.dtype)
    if not rms:
        assert bool(((mean.double().cpu() - m[:, 0]).abs() <= c * U * X.double().abs().mean(1) + U * m[:, 0].abs()).all())
    assert bool(((rstd.double().cpu() - r[:, 0]).abs() <= e_r[:, 0] * r[:, 0] if e_r.dim() else True).all())
    g = dY.double() * wd
    mg, mgx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    if rms:
        mg = torch.zeros_like(mg)
    e_mgx = c * U * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * e_x).mean(1, keepdim=True) + 2 * U * (g * xh).abs().mean(1, keepdim=True)
    e_mg = (c + 2) * U * g.abs().mean(1, keepdim=True)
    t = g - mg - xh * mgx
    e_t = 4 * U * (g.abs() + mg.abs() + (xh * mgx).abs()) + e_mg + e_x * mgx.abs() + xh.abs() * e_mgx + e_x * e_mgx
    close(dX, t * r, r * e_t + (e_r + 2 * U) * (t * r).abs(), X.dtype)
    terms = (dY.double() * xh).abs().sum(0)
    # a column: a workgroup's rows one after another, then the workgroups
    k = rows / 1024 + 1024 / 8 + 16
    close(dw, (dY.double() * xh).sum(0), k * U * terms + (dY.double().abs() * e_x).sum(0), w.dtype)
    if b is not None:
        close(db, dY.double().sum(0), k * U * dY.double().abs().sum(0), w.dtype)
    else:
        assert db is None
    return Y, dX, dw, db


TYPES = [(torch.float32, torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
         (torch.float16, torch.float32)]


@pytest.mark.parametrize("cols", [1, 7, 64, 100, 513, 1501, 2048, 4096, 6001, 8192, 12288, 16384])
@pytest.mark.parametrize("x,w", TYPES)
@pytest.mark.parametrize("rms,bias", [(False, True), (True, False)])
def test_every_width(slim, cols, x, w, rms, bias):
    X, dY, wt, b = data(37, cols, x, w, cols)
    check(slim, X, dY, wt, b if bias else None, 1e-5, rms)


@pytest.mark.parametrize("rows", [1, 2, 5, 16, 17, 64, 65, 1030, 5000])
@pytest.mark.parametrize("cols", [96, 1000, 1500, 4000])
@pytest.mark.parametrize("rms,bias", [(False, False), (True, True), (False, True)])
def test_every_height(slim, rows, cols, rms, bias):
    X, dY, wt, b = data(rows, cols, torch.bfloat16, torch.float32, rows)
    check(slim, X, dY, wt, b if bias else None, 1e-6, rms)


@pytest.mark.parametrize("x", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rms", [False, True])
def test_rows_longer_than_registers_hold(slim, x, rms):
    X, dY, wt, b = data(3, 70001, x, torch.float32, 3)
    check(slim, X, dY, wt, b, 1e-5, rms)


def test_a_large_mean_is_taken_off_before_squaring(slim):
    """Rows around 1000 with deviations of one: from the difference of two sums the variance would lose its digits."""
    X, dY, wt, b = data(64, 4096, torch.float32, torch.float32, 4)
    check(slim, X + 1000.0, dY, wt, b, 1e-5, False)


def test_gradients_are_differences_of_the_outputs(slim):
    """In 64 bits the formula's differences; the kernel's gradient agrees with them."""
    X, dY, wt, b = data(4, 50, torch.float32, torch.float32, 6)

    def f(x, w_, b_, rms):
        d = x - (0.0 if rms else x.mean(1, keepdim=True))
        return ((d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * w_ + b_) * dY.double()).sum()

    for rms in (False, True):
        _, dX, dw, db = check(slim, X, dY, wt, b, 1e-5, rms)
        h = 1e-5
        for i, j in ((0, 0), (3, 49), (2, 17)):
            for k, got in ((0, dX[i, j]), (1, dw[j]), (2, db[j])):
                at = [X.double(), wt.double(), b.double()]
                up, down = [v.clone() for v in at], [v.clone() for v in at]
                place = (i, j) if k == 0 else (j,)
                up[k][place] += h
                down[k][place] -= h
                diff = float(f(*up, rms) - f(*down, rms)) / (2 * h)
                # central differences: h^2 / 6 of the third derivative (below 1e3 here) and the sums' 1e-15 over h
                assert abs(float(got) - diff) <= 1e-7 + 1e-5 * max(1.0, abs(diff))


def test_special_rows(slim):
    """A row of one value has no deviations; one with a NaN or an infinity is NaN by itself and leaves the others alone."""
    X, dY, wt, b = data(6, 300, torch.float32, torch.float32, 7)
    X[1] = 3.0
    clean = slim.layer_norm(X.cuda(), wt.cuda(), b.cuda())
    assert torch.equal(clean[1].cpu(), b)
    check(slim, X, dY, wt, b, 1e-5, False)
    X[3, 5], X[4, 299] = float("nan"), float("inf")
    Y = slim.layer_norm(X.cuda(), wt.cuda(), b.cuda())
    assert torch.isnan(Y[3]).all() and torch.isnan(Y[4]).any()
    keep = [0, 1, 2, 5]
    assert torch.equal(Y[keep], clean[keep])
    zero = torch.zeros(2, 64, device="cuda")
    assert torch.equal(slim.layer_norm(zero, torch.ones(64).cuda(), None, 1e-5, rms=True), zero)


@pytest.mark.parametrize("x", [torch.float32, torch.float16])
def test_strides_and_alignment(slim, x):
    rows, cols = 70, 301
    X, dY, wt, b = data(rows, cols, x, x, 8)
    base = check(slim, X, dY, wt, b, 1e-5, False)

    def spread(v, first, gap):
        wide = torch.full((rows, cols + gap), float("nan"), dtype=x, device="cuda")
        wide[:, first:first + cols] = v.cuda()
        return wide[:, first:first + cols]

    off = torch.full((cols + 1,), float("nan"), dtype=x, device="cuda")
    off[1:] = wt.cuda()
    for first, gap in ((1, 1), (3, 7), (0, 2)):
        got = check(slim, X, dY, wt, b, 1e-5, False, (spread(X, first, gap), spread(dY, gap - first, gap), off[1:], b.cuda()))
        for p, q in zip(got, base):
            assert torch.equal(p, q)


def test_outputs_may_take_the_place_of_inputs(slim):
    from paper_2405_14917_amd import binding as B
    X, dY, wt, _ = data(50, 4096, torch.bfloat16, torch.bfloat16, 9)
    Xg, dYg, wg = X.cuda(), dY.cuda(), wt.cuda()
    Y, mean, rstd = slim.layer_norm(Xg, wg, stats=True)
    dX, dw, _ = slim.layer_norm_backward(dYg, Xg, wg, mean, rstd)
    p = lambda t: t.data_ptr()
    y2, d2, dw2 = Xg.clone(), dYg.clone(), torch.empty_like(dw)
    assert slim.lib.slim_layer_norm(slim.ctx, p(y2), B.BF16, 50, 4096, 4096, p(wg), None, B.BF16, 1e-5, 0, p(y2), 4096, None, None) == B.SLIM_OK
    assert slim.lib.slim_layer_norm_backward(slim.ctx, p(d2), p(Xg), B.BF16, 50, 4096, 4096, 4096, p(wg), B.BF16, p(mean), p(rstd), p(d2), 4096,
                                             p(dw2), None) == B.SLIM_OK
    assert torch.equal(y2, Y) and torch.equal(d2, dX) and torch.equal(dw2, dw)


def test_no_rows(slim):
    w = torch.ones(33, device="cuda")
    X = torch.empty((0, 33), device="cuda")
    Y, mean, rstd = slim.layer_norm(X, w, w, stats=True)
    dX, dw, db = slim.layer_norm_backward(X, X, w, mean, rstd, bias=True)
    assert Y.shape == dX.shape == (0, 33) and not dw.any() and not db.any()


def test_a_workspace_of_the_queried_size_is_enough():
    from paper_2405_14917_amd import binding
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    X, dY, w, _ = (t.cuda() for t in data(2000, 999, torch.float32, torch.float32, 10))
    for bias in (False, True):
        need = binding.layer_norm_backward_workspace(2000, 999, bias, torch.float32, ncu)
        for size, ok in ((need, True), (need - 256, False)):
            s = binding.Slim("cuda:0", workspace_bytes=size)
            try:
                Y, mean, rstd = s.layer_norm(X, w, stats=True)
                if ok:
                    s.layer_norm_backward(dY, X, w, mean, rstd, bias=bias)
                else:
                    with pytest.raises(binding.SlimError) as e:
                        s.layer_norm_backward(dY, X, w, mean, rstd, bias=bias)
                    assert e.value.status == binding.ERR_ALLOC
                torch.cuda.synchronize()
            finally:
                s.close()


def test_refusals(slim):
    from paper_2405_14917_amd import binding
    X, dY, w, b = (t.cuda() for t in data(4, 32, torch.float32, torch.float32, 11))
    _, mean, rstd = slim.layer_norm(X, w, stats=True)
    for bad in (lambda: slim.layer_norm(X, w[:31]), lambda: slim.layer_norm(X, w, b.half()), lambda: slim.layer_norm(X.t(), w),
                lambda: slim.layer_norm(X.cpu(), w), lambda: slim.layer_norm(X[0], w), lambda: slim.layer_norm(X, torch.ones(64).cuda()[::2]),
                lambda: slim.layer_norm_backward(dY.half(), X, w, mean, rstd), lambda: slim.layer_norm_backward(dY[:3], X, w, mean, rstd),
                lambda: slim.layer_norm_backward(dY, X, w, mean.double(), rstd), lambda: slim.layer_norm_backward(dY, X, w, mean, rstd[:3])):
        with pytest.raises(ValueError):
            bad()
    for bad, status in ((lambda: slim.layer_norm(X.double(), w.double()), binding.ERR_UNSUPPORTED),
                        (lambda: slim.layer_norm(X, w.half()), binding.ERR_UNSUPPORTED), (lambda: slim.layer_norm(X, w, eps=-1.0), binding.ERR_INVALID_ARG)):
        with pytest.raises(binding.SlimError) as e:
            bad()
        assert e.value.status == status


@pytest.mark.parametrize("cols,x", [(20000, torch.bfloat16), (9000, torch.float32), (12288, torch.float32), (70001, torch.float32)])
@pytest.mark.parametrize("rms,bias", [(False, True), (True, False)])
def test_gradients_of_long_rows_may_take_the_place_of_inputs(slim, cols, x, rms, bias):
    """Rows that the registers do not hold: the column sums are those of the inputs as they came, over dY as over X."""
    from paper_2405_14917_amd import binding as B
    rows = 40
    X, dY, wt, _ = data(rows, cols, x, torch.float32, cols)
    Xg, dYg, wg = X.cuda(), dY.cuda(), wt.cuda()
    _, dX, dw, db = check(slim, X, dY, wt, torch.zeros_like(wt) if bias else None, 1e-5, rms)
    _, mean, rstd = slim.layer_norm(Xg, wg, eps=1e-5, rms=rms, stats=True)
    p = lambda t: None if t is None else t.data_ptr()
    for over in ("dY", "X"):
        x2, dy2 = Xg.clone(), dYg.clone()
        out = dy2 if over == "dY" else x2
        dw2, db2 = torch.empty_like(dw), None if db is None else torch.empty_like(db)
        assert slim.lib.slim_layer_norm_backward(slim.ctx, p(dy2), p(x2), B.F32 if x == torch.float32 else B.BF16, rows, cols, cols, cols, p(wg), B.F32,
                                                 p(mean), p(rstd), p(out), cols, p(dw2), p(db2)) == B.SLIM_OK
        assert torch.equal(out, dX), over
        assert torch.equal(dw2, dw) and (db is None or torch.equal(db2, db)), over


@pytest.mark.parametrize("rows,cols,x", [(3001, 1501, torch.float32), (16384, 300, torch.bfloat16), (5000, 4096, torch.bfloat16), (700, 9000, torch.float32)])
def test_column_sums_are_rounded_at_their_end(slim, rows, cols, x):
    """Whole numbers whose sums over a workgroup's rows are exact in fp32 and over all rows are not: db is the exact sum, rounded once."""
    g = torch.Generator().manual_seed(rows)
    largest = 2 ** 17 if x == torch.float32 else 255                 # (all bits of the type)
    dY = torch.randint(-largest, largest + 1, (rows, cols), generator=g).double()
    if x == torch.bfloat16:
        dY *= 2.0 ** torch.randint(0, 9, (rows, 1), generator=g)    # (17 bits over the rows)
    dY += torch.where(dY > 0, largest, 0).double() * (x == torch.float32)      # sums that grow with the rows
    assert torch.equal(dY.to(x).double(), dY)
    X = torch.randn((rows, cols), generator=g).to(x)
    w = torch.ones(cols)
    _, mean, rstd = slim.layer_norm(X.cuda(), w.cuda(), stats=True)
    db = slim.layer_norm_backward(dY.to(x).cuda(), X.cuda(), w.cuda(), mean, rstd, bias=True)[2]
    assert torch.equal(db.cpu(), dY.sum(0).float())

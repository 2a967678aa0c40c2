"""The cross entropy over an 8-bit head without its logits, and its gradients, against their definition in 64 bits (fp8_reference.py).

Tolerances.  A logit's sum keeps 24 bits: e_z = (2 m / 8 + 16) 2^-23 sum |x| |w| (test_gpu_fp8_linear.py).  The log-sum-exp is off by no more than the
largest e_z of its classes, and by its own sum: 64 terms one after another and a tree, exponentials of 2^-22 each: 100 half steps of fp32 of 1; then
one rounding.  A probability is off by e_z + that + 8 half steps, relatively; dz by that and two roundings.  What the quantiser makes of dz: either
side of its range (test_gpu_linear_act.py), and the products' sums as there."""
import pytest
import torch

import fp8_reference as ref
from test_gpu_fp8_linear import numbers
from test_gpu_linear_act import U, check, gradient_range, product_of_range

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


def problem(V, m, t, x, seed=0):
    g = torch.Generator().manual_seed(seed)
    W = torch.randn((V, m), generator=g) * (2.0 / m ** 0.5) * torch.exp(0.3 * torch.randn((1, m), generator=g))
    X = torch.randn((t, m), generator=g)
    labels = torch.randint(0, V, (t,), generator=g)
    X += 0.5 * torch.rand((t, 1), generator=g) * W[labels] * m ** 0.5
    if t > 4:
        labels[t // 2], labels[1] = -100, V
    return W, X.to(x), labels, (torch.rand(t, generator=g) + 0.1) / t


def expected(W, X, labels):
    V, m = W.shape
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    z, e = A @ B.t(), (2 * m / 8 + 16) * 2.0 ** -23 * (A.abs() @ B.abs().t())
    live = (labels >= 0) & (labels < V)
    at = torch.where(live, labels, 0)[:, None]
    lse = torch.logsumexp(z, dim=1)
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], 0.0)
    e_lse = e.amax(1) + 100 * U
    e_loss = torch.where(live, e_lse + e.gather(1, at)[:, 0], 0.0)
    return B, z, e, live, at, lse, loss, e_lse, e_loss


def gradient_check(slim, V, m, t, x, dw, seed=0, labels_type=torch.int64):
    W, X, labels, dloss = problem(V, m, t, x, seed)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    lab = labels.to(labels_type).cuda()
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, lab, dloss.cuda(), dw)
    assert loss.dtype == torch.float32 and dX.dtype == x and dW.dtype == dw and dX.shape == X.shape and dW.shape == W.shape
    B, z, e, live, at, lse, want, e_lse, e_loss = expected(W, X, labels)
    check(loss, want, e_loss)
    assert torch.equal(loss, slim.head_loss(X.cuda(), q, s, lab))
    p = torch.exp(z - lse[:, None])
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    g = torch.where(live, dloss.double(), 0.0)[:, None]
    rel = e + e_lse[:, None] + 8 * U
    dz, e_dz = g * (p - one), g * (p * rel + 3 * U * (p - one).abs())
    lo, hi = dz - e_dz, dz + e_dz
    product_of_range(*gradient_range(lo, hi, "rows"), B, dX, False)
    least, most = gradient_range(lo, hi, "cols")
    product_of_range(least.t().contiguous(), most.t().contiguous(), ref.q_cols(X), dW, dw == torch.float32)
    assert not dX[~live.cuda()].any()
    return X, labels, dloss, (q, s, qt, st), loss, dX, dW


@pytest.mark.parametrize("V,m", [(1, 1), (5, 300), (127, 129), (130, 64), (1000, 257), (1537, 384)])
@pytest.mark.parametrize("t", [1, 2, 16, 17, 130])
@pytest.mark.parametrize("x,dw", [(torch.float16, torch.float16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_gradients(slim, V, m, t, x, dw):
    gradient_check(slim, V, m, t, x, dw)


@pytest.mark.parametrize("V,m,t", [(4100, 96, 700), (2050, 512, 1030), (33000, 64, 40), (40000, 128, 3), (8200, 3000, 1030), (5000, 130, 9000)])
def test_every_tile_and_several_pieces(slim, V, m, t):
    """Sizes that reach the tiles of both passes."""
    X, labels, dloss, W, loss, dX, dW = gradient_check(slim, V, m, t, torch.bfloat16, torch.float32)
    again = slim.head_loss_grad(X.cuda(), *W, labels.cuda(), dloss.cuda(), torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(again, (loss, dX, dW)))
    only = slim.head_loss_grad(X.cuda(), W[0], W[1], None, None, labels.int().cuda(), dloss.cuda(), torch.float32, dx=False)
    assert only[1] is None and torch.equal(only[2], dW) and torch.equal(only[0], loss)
    only = slim.head_loss_grad(X.cuda(), *W, labels.cuda(), dloss.cuda(), dw=False)
    assert only[2] is None and torch.equal(only[1], dX)


def test_several_pieces_with_odd_ends(slim):
    """Many tokens, an odd vocabulary."""
    gradient_check(slim, 2049, 65, 17000, torch.float16, torch.float16, labels_type=torch.int32)


def test_more_logits_than_are_kept(slim):
    """More than 64 Mi: the last classes' are computed again, and a piece ends where the kept ones do."""
    gradient_check(slim, 17001, 40, 4200, torch.float16, torch.float32)


@pytest.mark.parametrize("V,m,t", [(8300, 65, 17000), (601, 20, 66000), (1100, 20, 70000), (513, 20, 132000)])
def test_many_tokens(slim, V, m, t):
    """Three pieces, of 3584 classes and the rest; fewer logits kept than make a piece, in one piece and two: all losses, the gradients of some tokens and, at the
    pieces' ends, of some classes."""
    W, X, labels, dloss = problem(V, m, t, torch.float16, 5)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), torch.float32)
    classes = torch.tensor([c for c in (0, 1, 127, 128, 511, 512, 1023, 1024, 3583, 3584, 3585, 7167, 7168) if c < V] + [V - 1, int(labels[5]), int(labels[t - 1])])
    rows, cols = [], []
    for i in range(0, t, 2000):
        part = slice(i, min(t, i + 2000))
        B, z, e, live, at, lse, want, e_lse, e_loss = expected(W, X[part], labels[part])
        check(loss[part], want, e_loss)
        p = torch.exp(z - lse[:, None])
        off = p - torch.zeros_like(p).scatter_(1, at, 1.0)
        g = torch.where(live, dloss[part].double(), 0.0)[:, None]
        dz, e_dz = g * off, g * (p * (e + e_lse[:, None] + 8 * U) + 3 * U * off.abs())
        lo, hi = dz - e_dz, dz + e_dz
        some = torch.arange(0, len(lo), 397)
        rows.append((some + i, lo[some], hi[some]))
        cols.append((lo[:, classes], hi[:, classes]))
    at, lo, hi = (torch.cat(v) for v in zip(*rows))
    product_of_range(*gradient_range(lo, hi, "rows"), B, dX[at.cuda()], False)
    least, most = gradient_range(*(torch.cat(v) for v in zip(*cols)), "cols")
    product_of_range(least.t().contiguous(), most.t().contiguous(), ref.q_cols(X), dW[classes.cuda()], True)


@pytest.mark.parametrize("t", [1, 16, 40, 300, 2000])
@pytest.mark.parametrize("V", [700, 5003])
def test_losses(slim, t, V):
    W, X, labels, _ = problem(V, 320, t, torch.bfloat16, t)
    q, s = slim.fp8_quantize_weights(W.cuda(), transposed=False)
    loss = slim.head_loss(X.cuda(), q, s, labels.cuda())
    _, _, _, live, _, _, want, _, e = expected(W, X, labels)
    check(loss, want, e)
    assert torch.equal(loss, slim.head_loss(X.cuda(), q, s, labels.int().cuda())) and bool((loss[~live.cuda()] == 0).all())
    other = slim.head_loss(X.cuda(), q, s, torch.full_like(labels, 3).cuda())
    check(other, *(lambda r: (r[6], r[8]))(expected(W, X, torch.full_like(labels, 3))))


def test_gradients_are_differences_of_the_losses(slim):
    """The formula's gradient in 64 bits is its difference; the kernels' agrees with it to what e4m3 leaves: 2^-4 of each dz, as a bound on the sums."""
    V, m, t = 60, 40, 6
    W, X, labels, dloss = problem(V, m, t, torch.float16, 3)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    _, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), torch.float32)
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    live = (labels >= 0) & (labels < V)

    def f(a, b):
        z = a @ b.t()
        each = torch.logsumexp(z, 1) - z.gather(1, torch.where(live, labels, 0)[:, None])[:, 0]
        return float((torch.where(live, each, 0.0) * dloss.double()).sum())

    z = A @ B.t()
    dz = (torch.softmax(z, 1) - torch.zeros_like(z).scatter_(1, torch.where(live, labels, 0)[:, None], 1.0)) * torch.where(live, dloss.double(), 0.0)[:, None]
    h = 1e-5
    for i, j in ((0, 0), (3, 39), (5, 17)):
        up, down = A.clone(), A.clone()
        up[i, j] += h
        down[i, j] -= h
        diff = (f(up, B) - f(down, B)) / (2 * h)
        assert abs(float(dX[i, j]) - diff) <= 1e-7 + float(dz[i].abs() @ B[:, j].abs()) * (2.0 ** -4 + 2.0 ** -9) + abs(diff) * 2.0 ** -11
        v = int(labels[0]) if i == 0 else i
        up, down = B.clone(), B.clone()
        up[v, j] += h
        down[v, j] -= h
        diff = (f(A, up) - f(A, down)) / (2 * h)
        # (Qt(X) is another rounding than Q(X): 2^-4 of each as well)
        assert abs(float(dW[v, j]) - diff) <= 1e-7 + float(dz[:, v].abs() @ A[:, j].abs()) * (3 * 2.0 ** -4 + 2.0 ** -8)


@pytest.mark.parametrize("t", [3, 40, 300])
def test_tokens_without_a_label_and_gradients_of_zero(slim, t):
    V, m = 700, 200
    W, X, labels, dloss = problem(V, m, t, torch.bfloat16, 1)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    none = torch.full_like(labels, -1)
    bad = torch.full_like(dloss, float("nan"))                       # (not read there)
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, none.cuda(), bad.cuda())
    assert not loss.any() and not dX.any() and not dW.any()
    for far in (2 ** 31, 2 ** 40, -2 ** 63, V):
        some = labels.clone()
        some[0] = far
        loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, some.cuda(), dloss.cuda())
        assert float(loss[0]) == 0.0 and not dX[0].any()
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), torch.zeros_like(dloss).cuda())
    assert not dX.any() and not dW.any() and loss.any()


@pytest.mark.parametrize("t", [5, 40, 300])
def test_what_is_not_finite_stays_in_its_token(slim, t):
    V, m = 1000, 260
    W, X, labels, dloss = problem(V, m, t, torch.bfloat16, 2)
    labels[t - 1] = 3
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    clean = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), dw=False)
    X[t - 1, 7] = float("inf")
    loss, dX, _ = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), dw=False)
    assert torch.isnan(loss[t - 1]) and torch.isnan(dX[t - 1]).all()
    assert torch.equal(loss[:t - 1], clean[0][:t - 1]) and torch.equal(dX[:t - 1], clean[1][:t - 1])


@pytest.mark.parametrize("t", [4, 50, 300])
def test_large_logits(slim, t):
    """Logits of thousands: the probabilities are zeros and ones, the losses differences of two large numbers."""
    V, m = 900, 128
    W, X, labels, dloss = problem(V, m, t, torch.bfloat16, 5)
    W = W * 300.0
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    loss, dX, _ = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), dw=False)
    _, z, _, live, _, _, want, _, e = expected(W, X, labels)
    assert float(z.abs().max()) > 1000
    check(loss, want, e)
    assert torch.isfinite(dX).all()


def test_strides_and_other_rows(slim):
    """X inside a wider matrix; rows behind the last token and what lies between the rows of the gradients are left alone."""
    from paper_2405_14917_amd import binding as B
    V, m, t = 700, 130, 40
    W, X, labels, dloss = problem(V, m, t, torch.bfloat16, 6)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    lab, dl = labels.cuda(), dloss.cuda()
    want = slim.head_loss_grad(X.cuda(), q, s, qt, st, lab, dl)
    wide = torch.full((t, m + 7), float("nan"), dtype=X.dtype, device="cuda")
    wide[:, 3:3 + m] = X.cuda()
    got = slim.head_loss_grad(wide[:, 3:3 + m], q, s, qt, st, lab, dl)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    loss = torch.full((t + 1,), 7.0, device="cuda")
    dX, dW = torch.full((t + 1, m + 3), 7.0, dtype=X.dtype, device="cuda"), torch.full((V + 1, m + 5), 7.0, dtype=X.dtype, device="cuda")
    p = lambda v: v.data_ptr()
    Xg = X.cuda()
    assert slim.lib.slim_head_loss_grad(slim.ctx, p(Xg), B.BF16, t, m, p(q), q.stride(0), p(s), s.stride(0), p(qt), qt.stride(0), p(st), st.stride(0), V, m, p(lab),
                                        1, p(dl), p(loss), p(dX), m + 3, p(dW), B.BF16, m + 5) == B.SLIM_OK
    assert torch.equal(loss[:t], want[0]) and torch.equal(dX[:t, :m], want[1]) and torch.equal(dW[:V, :m], want[2])
    assert float(loss[t]) == 7 and bool((dX[t] == 7).all()) and bool((dX[:, m:] == 7).all()) and bool((dW[V] == 7).all()) and bool((dW[:, m:] == 7).all())


def test_no_tokens(slim):
    q, s, qt, st = slim.fp8_quantize_weights(torch.randn((300, 200), device="cuda"))
    X = torch.empty((0, 200), dtype=torch.bfloat16, device="cuda")
    lab, dl = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    assert slim.head_loss(X, q, s, lab).shape == (0,)
    loss, dX, dW = slim.head_loss_grad(X, q, s, qt, st, lab, dl, torch.float32)
    assert loss.shape == (0,) and dX.shape == (0, 200) and dW.shape == (300, 200) and not dW.any()


@pytest.mark.parametrize("V,m,t", [(1000, 256, 40), (5003, 130, 300), (2049, 65, 17000)])
def test_a_workspace_of_the_queried_size_is_enough(V, m, t):
    from paper_2405_14917_amd import binding
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    W, X, labels, dloss = problem(V, m, t, torch.bfloat16, 7)
    base = binding.Slim("cuda:0")
    w = base.fp8_quantize_weights(W.cuda())
    args = X.cuda(), *w, labels.cuda(), dloss.cuda()
    want = base.head_loss_grad(*args)
    need = binding.head_loss_grad_workspace(V, m, t, num_cus=ncu)
    c = binding.Slim("cuda:0", workspace_bytes=need)
    got = c.head_loss_grad(*args)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(c.head_loss(args[0], w[0], w[1], args[5]), want[0])
    torch.cuda.synchronize()
    c.close()
    small = binding.Slim("cuda:0", workspace_bytes=need // 2)
    with pytest.raises(binding.SlimError) as e:
        small.head_loss_grad(*args)
    assert e.value.status == binding.ERR_ALLOC
    small.close()
    base.close()


def test_refusals(slim):
    from paper_2405_14917_amd import binding
    W, X, labels, dloss = problem(300, 200, 5, torch.bfloat16)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    X, labels, dloss = X.cuda(), labels.cuda(), dloss.cuda()
    for bad in (lambda: slim.head_loss(X[:, :199], q, s, labels), lambda: slim.head_loss(X, q, s, labels[:4]), lambda: slim.head_loss(X, q, s, labels.float()),
                lambda: slim.head_loss(X, q, s[:2], labels), lambda: slim.head_loss(X, q, s, labels.cpu()), lambda: slim.head_loss(X[0], q, s, labels),
                lambda: slim.head_loss(X, q, s, torch.zeros(10, dtype=torch.int64, device="cuda")[::2]),
                lambda: slim.head_loss_grad(X, q, s, None, None, labels, dloss), lambda: slim.head_loss_grad(X, q, s, q, s, labels, dloss),
                lambda: slim.head_loss_grad(X, q, s, qt, st, labels, dloss.double()), lambda: slim.head_loss_grad(X, q, s, qt, st, labels, dloss[:4]),
                lambda: slim.head_loss_grad(X, q, s, qt, st, labels, dloss, dx=False, dw=False)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: slim.head_loss(X.float(), q, s, labels), lambda: slim.head_loss_grad(X, q, s, qt, st, labels, dloss, torch.float64)):
        with pytest.raises(binding.SlimError) as e:
            bad()
        assert e.value.status == binding.ERR_UNSUPPORTED

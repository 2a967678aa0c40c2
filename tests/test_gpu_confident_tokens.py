"""Cross entropy and gradients of tokens whose label's probability p is next to one: the loss, -ln p, and the label's own gradient, dloss (p - 1), are then
what the other classes' exponentials sum to, relatively as exact as they are.

Tolerances.  A logit is off by e_z (test_gpu_head_loss.py), a quotient of two exponentials relatively by twice that, the sum of the others by 100 half steps
of fp32 of its own, and 16 more for what follows.  With S the others' sum over the label's exponential, loss = ln(1 + S) and 1 - p = S / (1 + S), both off by no
more than S relatively.  Then as there: either side of what the quantiser makes of dz, and the products' sums."""
import pytest
import torch

import fp8_reference as ref
from test_gpu_head_loss import problem
from test_gpu_linear_act import U, gradient_range, product_of_range

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


def confident(V, m, t, x, seed=0):
    """Hidden states along their label's row of the head, 1 - p from some 1e-3 to 1e-9."""
    W, _, labels, dloss = problem(V, m, t, x, seed)
    labels = torch.randint(0, V, (t,), generator=torch.Generator().manual_seed(seed + 1))
    w = W[labels]
    lead = torch.linspace(14.0, 28.0, t)[:, None] if t > 1 else torch.tensor([[22.0]])
    X = w / (w * w).sum(1, keepdim=True) * lead + 0.3 * torch.randn((t, m), generator=torch.Generator().manual_seed(seed + 2)) / m ** 0.5
    return W, X.to(x), labels, dloss


def expected(W, X, labels):
    """Losses and their relative error; 1 - p and its; probabilities and theirs."""
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    z, e = A @ B.t(), (2 * W.shape[1] / 8 + 16) * 2.0 ** -23 * (A.abs() @ B.abs().t())
    at = labels[:, None]
    zl = z.gather(1, at)
    off = torch.exp(z - zl).scatter_(1, at, 0.0)
    S = off.sum(1)
    rel = 2 * e.amax(1) + 116 * U
    p = off / (1 + S)[:, None]
    return torch.log1p(S), S / (1 + S), p, rel, at, B


@pytest.mark.parametrize("V,m,t", [(1000, 256, 1), (1000, 256, 9), (700, 200, 300), (5003, 130, 600), (8200, 640, 1030), (16400, 256, 2100)])
@pytest.mark.parametrize("x,dw", [(torch.float16, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_losses_and_gradients(slim, V, m, t, x, dw):
    """Few tokens in one launch, and every tile of the product of logits."""
    W, X, labels, dloss = confident(V, m, t, x)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), dw)
    assert torch.equal(loss, slim.head_loss(X.cuda(), q, s, labels.cuda()))
    want, rest, p, rel, at, B = expected(W, X, labels)
    if t > 1:
        assert float(rest.min()) < 2e-7 and float(rest.max()) > 1e-5
    assert bool(((loss.double().cpu() - want).abs() <= (rel + U) * want).all())
    g = dloss.double()[:, None]
    dz = (g * p).scatter_(1, at, -g * rest[:, None])
    e = dz.abs() * rel[:, None]
    product_of_range(*gradient_range(dz - e, dz + e, "rows"), B, dX, False)
    least, most = gradient_range(dz - e, dz + e, "cols")
    product_of_range(least.t().contiguous(), most.t().contiguous(), ref.q_cols(X), dW, dw == torch.float32)


def test_logits_that_are_made_again(slim):
    """More than 64 Mi logits: the classes behind the first pieces, whose gradients are formed at the end of the product."""
    V, m, t = 17001, 40, 4200
    W, X, labels, dloss = confident(V, m, t, torch.float16, 3)
    labels[:] = torch.randint(15900, V, (t,), generator=torch.Generator().manual_seed(8))
    w = W[labels]
    X = (w / (w * w).sum(1, keepdim=True) * torch.linspace(16.0, 30.0, t)[:, None]).half()
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), torch.float32)
    least, most = [], []
    classes = torch.arange(15900, V, 3)
    for i in range(0, t, 1024):
        part = slice(i, min(t, i + 1024))
        want, rest, p, rel, at, B = expected(W, X[part], labels[part])
        assert bool(((loss[part].double().cpu() - want).abs() <= (rel + U) * want).all())
        g = dloss[part].double()[:, None]
        dz = (g * p).scatter_(1, at, -g * rest[:, None])
        e = dz.abs() * rel[:, None]
        some = torch.arange(0, len(dz), 61)
        product_of_range(*gradient_range((dz - e)[some], (dz + e)[some], "rows"), B, dX[(some + i).cuda()], False)
        a, b = gradient_range((dz - e)[:, classes], (dz + e)[:, classes], "cols")
        least.append(a)
        most.append(b)
    least, most = torch.cat(least), torch.cat(most)
    product_of_range(least.t().contiguous(), most.t().contiguous(), ref.q_cols(X), dW[classes.cuda()], True)


@pytest.mark.parametrize("t", [3, 40, 300])
@pytest.mark.parametrize("V", [1, 17, 65, 129, 257, 400])
def test_labels_alone_in_their_tile(slim, V, t):
    """A last tile of one class, which is every token's label: nothing else in it has an exponential.  A vocabulary of one has no loss."""
    W, X, _, dloss = problem(V, 130, t, torch.bfloat16, 2)
    labels = torch.full((t,), V - 1)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    loss, dX, dW = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), torch.float32)
    want, rest, p, rel, at, B = expected(W, X, labels)
    assert bool(((loss.double().cpu() - want).abs() <= (rel + U) * want).all())
    g = dloss.double()[:, None]
    dz = (g * p).scatter_(1, at, -g * rest[:, None])
    e = dz.abs() * rel[:, None]
    product_of_range(*gradient_range(dz - e, dz + e, "rows"), B, dX, False)
    if V == 1:
        assert not loss.any() and not dX.any() and not dW.any()


@pytest.mark.parametrize("t", [5, 300])
def test_losses_below_the_last_digit_of_one(slim, t):
    """Losses down to fp32's smallest numbers, not zero."""
    V, m = 900, 64
    W, X, labels, dloss = confident(V, m, t, torch.float16, 4)
    w = W[labels]
    X = (w / (w * w).sum(1, keepdim=True) * torch.linspace(70.0, 130.0, t)[:, None]).half()
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    loss = slim.head_loss_grad(X.cuda(), q, s, qt, st, labels.cuda(), dloss.cuda(), dw=False)[0]
    assert torch.equal(loss, slim.head_loss(X.cuda(), q, s, labels.cuda()))
    want, _, _, rel, _, _ = expected(W, X, labels)
    assert float(want.max()) < 2.0 ** -24 and float(want.min()) < 1e-25
    assert bool(((loss.double().cpu() - want).abs() <= (rel + U) * want + 2.0 ** -149).all()) and bool((loss > 0).all())

"""Cross entropy over more logits than are kept, with a contraction of many blocks: the classes behind the kept ones in tiles of 256 x 256 whose ends form the gradients
(test_gradient_tiles_host.py has the launches of these sizes).  All losses, the gradients of some tokens and of classes at the pieces' ends.

Tolerances.  Number by number as in test_gpu_confident_tokens.py.  In the norm: half a step of the output's type; 2^-10 for what the e4m3 matrix cores drop
(test_gpu_error_norms.py; not of fp32 outputs); a logit is in truth off by less than 2^-16, what is left of independent errors, so that fewer than one number in 2^12 is
quantised to the other side of a border, a step of 2^-3 of it at most: 2^-9.  Exponentials have no results below 2^-126, nor losses and gradients digits below 2^-149:
many of these tokens are that sure."""
import pytest
import torch

import fp8_reference as ref
from test_gpu_head_loss import problem
from test_gpu_linear_act import HALF, U, gradient_range, product_of_range

pytestmark = pytest.mark.gpu

# (classes, width, tokens, pieces' ends): one piece kept and one made again; one kept and two, the last one's tiles ragged both ways
SIZES = [(40000, 2560, 2048, (32768,)), (16500, 2600, 8200, (7680, 15360))]


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


@pytest.mark.parametrize("V,m,t,ends", SIZES)
def test_large_tiles_of_logits_made_again(slim, V, m, t, ends):
    x = torch.bfloat16
    W, X, labels, dloss = problem(V, m, t, x, 11)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    Xg, lab, dl = X.cuda(), labels.cuda(), dloss.cuda()
    loss, dX, dW = slim.head_loss_grad(Xg, q, s, qt, st, lab, dl, torch.float32)
    print("gradients done", flush=True)
    A, B = ref.q_rows(X), ref.quantize(W, ref.B, ref.B)[2]
    Ag, Bt = A.cuda(), B.cuda().t().contiguous()
    size = Bt.abs()
    classes = sorted({c + k for c in (0, 128, 256, *ends, V) for k in (-129, -128, -1, 0, 1, 127, 255) if 0 <= c + k < V} | set(labels[5:300:7].tolist()))
    tokens = sorted({0, 1, 127, 128, 255, 256, t - 1, t - 9, t // 2} | set(range(2, t, 131)))
    cols = torch.tensor(classes)
    lows, highs, mids, row_lo, row_hi, row_mid = [], [], [], [], [], []
    for i in range(0, t, 1024):
        part = slice(i, min(t, i + 1024))
        z, e = Ag[part] @ Bt, (2 * m / 8 + 16) * 2.0 ** -23 * (Ag[part].abs() @ size)
        live = (lab[part] >= 0) & (lab[part] < V)
        at = torch.where(live, lab[part], 0)[:, None]
        off = torch.exp(z - z.gather(1, at)).scatter_(1, at, 0.0)
        S, rel = off.sum(1), 2 * e.amax(1) + 116 * U
        want = torch.where(live, torch.log1p(S), 0.0)
        assert bool(((loss[part].double() - want).abs() <= (rel + U) * want + 2.0 ** -149).all())
        g = torch.where(live, dl[part].double(), 0.0)[:, None]
        dz = (g * off / (1 + S)[:, None]).scatter_(1, at, -g * (S / (1 + S))[:, None])
        err = dz.abs() * rel[:, None] + g * 2.0 ** -126
        some = torch.tensor([k - i for k in tokens if i <= k < i + len(dz)])
        for to, v in ((row_mid, dz), (row_lo, dz - err), (row_hi, dz + err)):
            to.append(v[some.cuda()].cpu())
        for to, v in ((mids, dz), (lows, dz - err), (highs, dz + err)):
            to.append(v[:, cols.cuda()].cpu())
        print("tokens to", i + len(dz), flush=True)
    mid, lo, hi = (torch.cat(v) for v in (row_mid, row_lo, row_hi))
    got = dX[torch.tensor(tokens).cuda()]
    product_of_range(*gradient_range(lo, hi, "rows"), B, got, False)
    exact = ref.q_rows(mid) @ B
    assert float((got.double().cpu() - exact).norm() / exact.norm()) <= HALF[x] + 2.0 ** -10 + 2.0 ** -9
    mid, lo, hi = (torch.cat(v) for v in (mids, lows, highs))
    got, xt = dW[cols.cuda()], ref.q_cols(X)
    least, most = gradient_range(lo, hi, "cols")
    product_of_range(least.t().contiguous(), most.t().contiguous(), xt, got, True)
    exact = ref.q_cols(mid).t() @ xt
    assert float((got.double().cpu() - exact).norm() / exact.norm()) <= 2.0 ** -9
    # again, and each gradient alone: the same bits
    again = slim.head_loss_grad(Xg, q, s, qt, st, lab, dl, torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(again, (loss, dX, dW)))
    only = slim.head_loss_grad(Xg, q, s, None, None, lab.int(), dl, torch.float32, dx=False)
    assert only[1] is None and torch.equal(only[2], dW) and torch.equal(only[0], loss)
    only = slim.head_loss_grad(Xg, q, s, qt, st, lab, dl, dw=False)
    assert only[2] is None and torch.equal(only[1], dX) and torch.equal(slim.head_loss(Xg, q, s, lab), loss)


@pytest.mark.parametrize("V,m,t", [(17001, 40, 4200), (1100, 20, 70000)])
def test_each_gradient_alone_over_several_pieces(slim, V, m, t):
    """Medium tiles made again, with and without a piece that is kept."""
    W, X, labels, dloss = problem(V, m, t, torch.float16, 12)
    q, s, qt, st = slim.fp8_quantize_weights(W.cuda())
    Xg, lab, dl = X.cuda(), labels.cuda(), dloss.cuda()
    loss, dX, dW = slim.head_loss_grad(Xg, q, s, qt, st, lab, dl)
    again = slim.head_loss_grad(Xg, q, s, qt, st, lab, dl)
    assert all(torch.equal(a, b) for a, b in zip(again, (loss, dX, dW)))
    only = slim.head_loss_grad(Xg, q, s, None, None, lab, dl, dx=False)
    assert only[1] is None and torch.equal(only[2], dW) and torch.equal(only[0], loss)
    only = slim.head_loss_grad(Xg, q, s, qt, st, lab, dl, dw=False)
    assert only[2] is None and torch.equal(only[1], dX)

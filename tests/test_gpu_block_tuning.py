"""The step that tunes a feed-forward block in 8 bits and its head against labels (tuning.py): all of its operators together, eagerly and captured."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def problem(t, dtype, seed=0, width=256, inner=640, V=1003):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    up, down, head = r(inner, width) * width ** -0.5, r(width, inner) * inner ** -0.5, r(V, width) * width ** -0.5
    X, R = 0.5 * r(t, width), r(t, width)
    labels = torch.randint(0, V, (t,), generator=g)
    if t > 8:
        labels[t // 2] = -100
    vectors = 1 + 0.1 * r(width), 0.1 * r(width), 1 + 0.1 * r(width), 0.1 * r(width), 0.1 * r(inner), 0.1 * r(width)
    return [v.cuda() for v in (up, down, head)], X.to(dtype).cuda(), R.to(dtype).cuda(), labels.cuda(), [v.cuda() for v in vectors]


def block(slim, W, v, bias=True, **more):
    from paper_2405_14917_amd import tuning
    b = (lambda x: x) if bias else (lambda x: None)
    return tuning.BlockTuning(slim, *W, (v[0], b(v[1])), (v[2], b(v[3])), b(v[4]), b(v[5]), **more)


def flat(grads):
    return [v for k in sorted(grads) for v in (grads[k] if isinstance(grads[k], tuple) else (grads[k],)) if v is not None]


@pytest.mark.parametrize("t", [1, 16, 300])
@pytest.mark.parametrize("act,rms,bias", [("silu", True, False), ("gelu", False, True)])
def test_the_gradients_are_those_of_the_block(t, act, rms, bias):
    """Against autograd in fp64 of the same block without its roundings to e4m3.  Such a rounding is off by at most 2^-4 of a number, 2^-4 / sqrt(3) in the
    root mean square where its place between two numbers is random, and that is what it adds to a sum's norm.  Twelve of them meet in the longest path,
    that of `up`: dz, head, dH, down, dZ, the norm's output; those of the activation's slope (2), of the second norm (2), of the probabilities
    (2): 2^-4 sqrt(12 / 3)."""
    from paper_2405_14917_amd import binding
    slim = binding.Slim("cuda:0")
    W, X, R, labels, v = problem(t, torch.float16)
    b = block(slim, W, v, bias, act=act, rms=rms)
    dloss = torch.full((t,), 1.0 / t, device="cuda")
    loss, g, norm = b.gradients(X, R, labels, dloss)

    leaf = lambda x: x.double().requires_grad_()
    up, down, head = map(leaf, W)
    x, r = leaf(X), R.double()
    w1, b1, w2, b2, ub, db = map(leaf, v)

    def normed(h, w, c):
        d = h if rms else h - h.mean(1, keepdim=True)
        y = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * w
        return y + c if bias else y

    h = x + r
    z = normed(h, w1, b1) @ up.t() + (ub if bias else 0.0)
    u = z * torch.sigmoid(z) if act == "silu" else z * torch.special.ndtr(z)
    h2 = h + u @ down.t() + (db if bias else 0.0)
    lnp = torch.log_softmax(normed(h2, w2, b2) @ head.t(), 1)
    live = labels >= 0
    each = torch.where(live, -lnp.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0)
    (each * dloss.double()).sum().backward()
    assert float((loss.double() - each.detach()).norm() / each.detach().norm()) < 0.125
    pairs = [(g["X"], x), (g["up"], up), (g["down"], down), (g["head"], head), (g["norm1"][0], w1), (g["norm2"][0], w2)]
    if bias:
        pairs += [(g["norm1"][1], b1), (g["norm2"][1], b2), (g["up_bias"], ub), (g["down_bias"], db)]
    else:
        assert g["norm1"][1] is None and g["up_bias"] is None
    for got, of in pairs:
        assert got.shape == of.shape
        assert float((got.double() - of.grad).norm() / of.grad.norm()) < 0.125
    parameters = [q for q, o in pairs[1:]]
    want = torch.sqrt(sum((q.double() ** 2).sum() for q in parameters))
    assert abs(float(norm) - float(want)) <= 2.0 ** -23 * float(want)
    # scaled down together, the gradient of the inputs not
    loss2, g2, norm2 = b.gradients(X, R, labels, dloss, limit=0.5 * float(norm))
    assert torch.equal(loss2, loss) and torch.equal(norm2, norm) and torch.equal(g2["X"], g["X"])
    for a, c in zip(flat({k: g2[k] for k in g2 if k != "X"}), flat({k: g[k] for k in g if k != "X"})):
        assert bool(((a.double() - 0.5 * c.double()).abs() <= 2.0 ** -22 * c.double().abs() + 2.0 ** -140).all())
    torch.cuda.synchronize()
    slim.close()


@pytest.mark.parametrize("t", [1, 40])
def test_serving_and_training_agree(t):
    """The loss of validate is that of gradients; the logits are those whose cross entropy it is."""
    from paper_2405_14917_amd import binding
    slim = binding.Slim("cuda:0")
    W, X, R, labels, v = problem(t, torch.bfloat16)
    b = block(slim, W, v)
    loss = b.gradients(X, R, labels, torch.ones(t, device="cuda"))[0]
    assert torch.equal(b.validate(X, R, labels), loss)
    z = b.logits(X, R).double()
    live = labels >= 0
    want = torch.where(live, torch.logsumexp(z, 1) - z.gather(1, labels.clamp(min=0)[:, None])[:, 0], 0.0)
    # (both in fp32 with 24 bits: sums of 256 products of a size of 40 at most, in another order)
    assert float((loss.double() - want).abs().max()) <= 2 * (2 * 256 / 8 + 16) * 2.0 ** -23 * 40
    alone = b.logits(X, None)
    assert alone.shape == z.shape and not torch.equal(alone.double(), z)
    torch.cuda.synchronize()
    slim.close()


@pytest.mark.parametrize("t", [1, 16, 200])
def test_captured_into_a_graph(t):
    """The whole step under capture in a workspace of the queried size, another graph in the same workspace beside it; every replay, with new inputs, new
    weights and eager work between, is the eager result to the last bit."""
    from paper_2405_14917_amd import binding, tuning
    W, X, R, labels, v = problem(t, torch.bfloat16)
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    dloss = torch.full((t,), 1.0 / t, device="cuda")
    eager = block(binding.Slim("cuda:0"), W, v)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        slim = binding.Slim("cuda:0", workspace_bytes=tuning.block_workspace_query(1003, 256, 640, t, num_cus=ncu))
        b = block(slim, W, v)
        b.gradients(X, R, labels, dloss, 0.1)
        b.logits(X, R)
    stream.synchronize()
    graph, serve = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loss, g, norm = b.gradients(X, R, labels, dloss, 0.1)
    with torch.cuda.graph(serve, stream=stream):
        z = b.logits(X, R)
    for seed in range(1, 5):
        W2, X2, R2, l2, _ = problem(t, torch.bfloat16, seed)
        X.copy_(X2), R.copy_(R2), labels.copy_(l2)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            b.store(*W2)
        stream.synchronize()
        eager.store(*W2)
        want, gw, nw = eager.gradients(X, R, labels, dloss, 0.1)
        zw = eager.logits(X, R)
        torch.cuda.synchronize()
        for first in (graph, serve) if seed % 2 else (serve, graph):
            first.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want) and torch.equal(norm, nw) and torch.equal(z, zw)
        assert all(torch.equal(a, c) for a, c in zip(flat(g), flat(gw)))
    del graph, serve
    torch.cuda.synchronize()
    slim.close()
    eager.slim.close()


def test_parameters_that_require_gradients():
    from paper_2405_14917_amd import binding
    slim = binding.Slim("cuda:0")
    W, X, R, labels, v = problem(5, torch.bfloat16)
    P = torch.nn.Parameter
    plain, b = block(slim, W, v), block(slim, [P(w) for w in W], [P(x) for x in v])
    dloss = torch.full((5,), 0.2, device="cuda")
    loss, g, n = plain.gradients(X, R, labels, dloss)
    loss2, g2, n2 = b.gradients(X, R, labels, dloss)
    assert torch.equal(loss, loss2) and torch.equal(n, n2) and all(torch.equal(a, c) for a, c in zip(flat(g), flat(g2)))
    with torch.no_grad():
        assert torch.equal(b.validate(X, R, labels), loss)
    for call in (lambda: b.hidden(X, R), lambda: b.validate(X, R, labels), lambda: plain.hidden(X.clone().requires_grad_(), R)):
        with pytest.raises(ValueError, match="graph"):
            call()
    torch.cuda.synchronize()
    slim.close()

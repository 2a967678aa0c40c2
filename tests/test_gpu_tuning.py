"""The step that tunes a norm and an 8-bit head against a teacher (tuning.py): the calls in their order, and captured into a graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def problem(t, V, m, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    W, X = r(V, m) * 0.05, r(t, m)
    T = (X @ W.t() * 1.5 + 0.3 * r(t, V))
    teacher, index = torch.topk(T, 12, dim=1)
    return W.cuda(), X.to(dtype).cuda(), (1 + 0.1 * r(m)).cuda(), (0.1 * r(m)).cuda(), index.cuda(), teacher.cuda(), torch.logsumexp(T.double(), 1).float().cuda()


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("t", [1, 40, 300])
def test_gradients_lower_the_loss(rms, t):
    """A step along the gradients of norm and head lowers the divergence by about what they promise."""
    from paper_2405_14917_amd import binding, tuning
    slim = binding.Slim("cuda:0")
    W, X, w, b, index, teacher, lse = problem(t, 1003, 256, torch.bfloat16)
    head = tuning.HeadTuning(slim, W, w, None if rms else b, rms=rms)
    dloss = torch.full((t,), 1.0 / t, device="cuda")
    loss, g = head.gradients(X, index, teacher, dloss, lse)
    assert torch.equal(loss, head.validate(X, index, teacher, lse))
    assert (g["bias"] is None) == rms and g["head"].shape == W.shape and g["X"].shape == X.shape
    only, g2 = head.gradients(X, index, teacher, dloss, lse, head_grad=False)
    assert g2["head"] is None and torch.equal(only, loss) and torch.equal(g2["weight"], g["weight"])
    before = float(loss.mean())
    size = float(g["weight"].double().norm()) if rms else float(torch.sqrt(g["weight"].double().norm() ** 2 + g["bias"].double().norm() ** 2))
    h = 0.05 * before / size ** 2                                # 5 % of the loss by its first derivative
    head.weight = w - h * g["weight"]
    if not rms:
        head.bias = b - h * g["bias"]
    after = float(head.validate(X, index, teacher, lse).mean())
    assert 0.0 < before - after < 0.1 * before, (before, after)
    head.weight, head.bias = w, None if rms else b
    h = 0.2 * before / float(g["head"].double().norm()) ** 2      # (a step that the head's three digits can show)
    head.store(W - h * g["head"])
    assert float(head.validate(X, index, teacher, lse).mean()) < before
    torch.cuda.synchronize()
    slim.close()


@pytest.mark.parametrize("t", [1, 16, 200])
def test_captured_into_a_graph(t):
    """The whole step under capture, in a workspace of the queried size; every replay, with new inputs and eager work between, is the eager
    result to the last bit."""
    from paper_2405_14917_amd import binding, tuning
    V, m = 1003, 384
    W, X, w, b, index, teacher, lse = problem(t, V, m, torch.bfloat16)
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    dloss = torch.full((t,), 1.0 / t, device="cuda")
    eager = tuning.HeadTuning(binding.Slim("cuda:0"), W, w, b)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        slim = binding.Slim("cuda:0", workspace_bytes=tuning.workspace_query(V, m, t, num_cus=ncu))
        head = tuning.HeadTuning(slim, W, w, b)
        head.gradients(X, index, teacher, dloss, lse)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loss, g = head.gradients(X, index, teacher, dloss, lse)
    for seed in range(1, 5):
        _, X2, _, _, i2, t2, l2 = problem(t, V, m, torch.bfloat16, seed)
        X.copy_(X2), index.copy_(i2), teacher.copy_(t2), lse.copy_(l2)
        want, gw = eager.gradients(X, index, teacher, dloss, lse)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want)
        for k in gw:
            assert torch.equal(g[k], gw[k]), k
    del graph
    torch.cuda.synchronize()
    slim.close()
    eager.slim.close()


@pytest.mark.parametrize("t", [16, 200])
def test_new_weights_between_replays(t):
    """Captured gradients, an update of the head, other allocations, a replay: the loop of a tuning step."""
    from paper_2405_14917_amd import binding, tuning
    V, m = 1003, 384
    W, X, w, b, index, teacher, lse = problem(t, V, m, torch.bfloat16)
    ncu = torch.cuda.get_device_properties(0).multi_processor_count
    dloss = torch.full((t,), 1.0 / t, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        slim = binding.Slim("cuda:0", workspace_bytes=tuning.workspace_query(V, m, t, num_cus=ncu))
        head = tuning.HeadTuning(slim, W, w, b)
        head.gradients(X, index, teacher, dloss, lse)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        loss, g = head.gradients(X, index, teacher, dloss, lse)
    place = [v.data_ptr() for v in (head.q, head.s, head.qt, head.st)]
    for seed in range(1, 5):
        W2 = problem(1, V, m, torch.bfloat16, seed)[0]
        with torch.cuda.stream(stream):
            head.store(W2)
        stream.synchronize()
        assert [v.data_ptr() for v in (head.q, head.s, head.qt, head.st)] == place
        other = tuning.HeadTuning(binding.Slim("cuda:0"), W2, w, b)
        want, gw = other.gradients(X, index, teacher, dloss, lse)
        junk = [torch.full_like(v.view(torch.uint8), 0x7f) for v in (head.q, head.qt, other.q, other.qt)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want)
        for k in gw:
            assert torch.equal(g[k], gw[k]), k
        other.slim.close()
        del junk
    with torch.cuda.stream(stream), pytest.raises(ValueError):
        head.store(W[:1000])
    del graph
    torch.cuda.synchronize()
    slim.close()


def test_parameters():
    """A norm's weight that requires a gradient: the step, whose gradients are its results, takes it; serving does under no_grad and refuses to lose the
    gradient elsewhere."""
    from paper_2405_14917_amd import binding, tuning
    slim = binding.Slim("cuda:0")
    W, X, w, b, index, teacher, lse = problem(5, 300, 256, torch.bfloat16)
    dloss = torch.full((5,), 0.2, device="cuda")
    plain = tuning.HeadTuning(slim, W, w, b)
    head = tuning.HeadTuning(slim, torch.nn.Parameter(W), torch.nn.Parameter(w), torch.nn.Parameter(b))
    loss, g = plain.gradients(X, index, teacher, dloss, lse)
    loss2, g2 = head.gradients(X, index, teacher, dloss, lse)
    assert torch.equal(loss, loss2) and all(torch.equal(g[k], g2[k]) for k in g)
    with torch.no_grad():
        assert torch.equal(head.validate(X, index, teacher, lse), loss)
        head.store(torch.nn.Parameter(W))
    for call in (lambda: head.logits(X), lambda: head.validate(X, index, teacher, lse), lambda: plain.logits(X.clone().requires_grad_())):
        with pytest.raises(ValueError, match="graph"):
            call()
    torch.cuda.synchronize()
    slim.close()

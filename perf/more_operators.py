"""The operators of a block around quantised layers and of its training step, as a list of cases that can be timed and compared.

  add_norm       the residual stream takes a branch's output and is normalised (with or without the mean), in 16 or 32 bits, in e4m3 numbers
                 with a scale for every 128 channels, or both: a token or a prompt
  add_norm_grad  the same as a training step: both outputs, and the gradients of stream and branch, weight and bias
  linear         the 8-bit linear layer with bias, activation and residual, from activations of 16 bits or from the e4m3 form above
  linear_grad    its backward pass: the gradients of activations, weights and bias, from that of the outputs and the values before the activation
  head           the cross entropy of the label in the softmax of an 8-bit head's outputs, token by token (validation)
  head_grad      the same with the gradients of hidden states and head (training)
  clip           the norm of all gradients of a model together, and the gradients scaled down where it is above a limit

Where `own` is false the operators are computed in their plain form.  What is computed, in both:

quantiser    a = max |x| over a block's finite elements; s the smallest power of two, at least 2^-126, with a <= 448 s; stored are
             the e4m3 numbers nearest to x / s (ties to even; NaN for an x that is not finite) and the byte log2(s) + 127
add_norm     h = x + r, rounded to their type; mu, v over a row of h, hh = (h - mu) / sqrt(v + eps), y = hh w + b, rounded; without the mean: mu = 0,
             v = mean h^2; the e4m3 form is that of the rounded y.  dx = dr = dh + (g - mean g - hh mean(g hh)) / sqrt(v + eps) for g = dy w
             (no mean g without the mean; dh: the gradient that reaches h past the norm);  dw = sum dy hh, db = sum dy
linear       z = Q(x) W^T + bias, y = act(z) + residual;  act: relu, gelu(z) = z Phi(z), silu(z) = z / (1 + exp(-z)), or none
             dz = dy act'(z), rounded to dy's type;  Q(dz) W with blocks along the outputs, Qt(dz)^T Qt(x) with blocks of 128 tokens, dbias = sum dy act'(z)
head         z = Q(x) W^T, loss = ln sum exp z - z[label], 0 for a label outside the vocabulary;  dz = dloss (softmax z - [label]), none for such
             a label;  dx = Q(dz) W with blocks along the vocabulary,  dW = Qt(dz)^T Qt(x) with blocks of 128 tokens
clip         n = sqrt(sum of all squares);  g min(1, limit / n)
"""
import math

import torch

own = False

BLOCK = 128
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
E4M3 = torch.float8_e4m3fn
E8M0 = torch.float8_e8m0fnu
EPS = 1e-5
RUN = 4                  # outlier channels come in runs of this length


def listed():
    return [
        # decoding: the stream of one token in front of a projection that is kept in 8 bits
        dict(name="add_norm_1x4096", kind="add_norm", rows=1, cols=4096, x="bf16", w="bf16", rms=True, bias=False, y=False, q=True),
        # a training step of 8 samples of 2048 tokens; the product takes the 8-bit form, its backward pass the 16-bit one
        dict(name="add_norm_grad_16384x4096", kind="add_norm_grad", rows=16384, cols=4096, x="bf16", w="bf16", rms=True, bias=False, y=True, q=True),
        # odd rows and columns, with the mean and a bias
        dict(name="add_norm_grad_3001x1501", kind="add_norm_grad", rows=3001, cols=1501, x="f16", w="f32", rms=False, bias=True, y=True, q=False),
        # decoding: one token through the widening layer of a feed-forward block
        dict(name="linear_11008x4096_t1", kind="linear", n=11008, m=4096, t=1, x="e4m3", y="bf16", act="silu", bias=True, res=False, z=False),
        # a prompt through the layer that ends the block: bias and residual
        dict(name="linear_4096x11008_t2048", kind="linear", n=4096, m=11008, t=2048, x="bf16", y="bf16", act="none", bias=True, res=True, z=False),
        # a ragged layer in training: the values before the activation are kept
        dict(name="linear_1000x1504_t301", kind="linear", n=1000, m=1504, t=301, x="e4m3", y="f16", act="gelu", bias=True, res=False, z=True),
        # the gradients of the widening layer for two samples of 2048 tokens
        dict(name="linear_grad_11008x4096_t4096", kind="linear_grad", n=11008, m=4096, t=4096, x="bf16", act="gelu", bias="f32"),
        # validation of one token with a head of 32000 classes
        dict(name="head_32000x4096_t1", kind="head", V=32000, m=4096, t=1, x="bf16"),
        # a training sample of 2048 tokens
        dict(name="head_grad_32000x4096_t2048", kind="head_grad", V=32000, m=4096, t=2048, x="bf16"),
        # an odd, larger vocabulary, ragged width
        dict(name="head_grad_50257x1501_t301", kind="head_grad", V=50257, m=1501, t=301, x="f16"),
        # the gradients of one small layer
        dict(name="clip_1x256", kind="clip", layers=1, width=256, inner=704, x="bf16", limit=1.0),
        # the gradients of two layers of the benchmark's width
        dict(name="clip_2x4096", kind="clip", layers=2, width=4096, inner=11008, x="bf16", limit=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case; none has more work than the largest of its kind in the list."""
    kind = rng.choice(["add_norm", "add_norm_grad", "add_norm_grad", "linear", "linear", "linear", "linear_grad", "linear_grad", "head",
                       "head_grad", "head_grad", "clip"])
    x = rng.choice(["f16", "bf16", "bf16"])
    if kind in ("add_norm", "add_norm_grad"):
        while True:
            c = dict(kind=kind, rows=_log(rng, 1, 32768), cols=_log(rng, 64, 16384), x=rng.choice(["f16", "bf16", "f32"]), w="f32",
                     rms=rng.random() < 0.5, bias=rng.random() < 0.5)
            c["w"] = rng.choice([c["x"], "f32"])
            c["y"], c["q"] = rng.choice([(True, False), (False, True), (True, True)])
            if rng.random() < 0.6:
                c["cols"] = max(64, c["cols"] // 64 * 64)
            if c["rows"] * c["cols"] <= 16384 * 4096:
                return c
    if kind in ("linear", "linear_grad"):
        while True:
            c = dict(kind=kind, n=_log(rng, 128, 28672), m=_log(rng, 128, 11008), t=_log(rng, 1 if kind == "linear" else 32, 8192), x=x,
                     act=rng.choice(["none", "relu", "gelu", "gelu", "silu", "silu"]))
            if kind == "linear":
                c.update(y=rng.choice([x, x, "f32"]), bias=rng.random() < 0.5, res=rng.random() < 0.5, z=rng.random() < 0.3)
                if rng.random() < 0.5:
                    c["x"] = "e4m3"
            else:
                c.update(bias=rng.choice(["none", "f32", x]))
            if rng.random() < 0.5:                      # half of the layers have whole blocks
                c.update(n=max(128, c["n"] // 128 * 128), m=max(128, c["m"] // 128 * 128))
            if work(c)["flops"] <= 0.7e12 and c["n"] * c["m"] <= 28672 * 8192:
                return c
    if kind in ("head", "head_grad"):
        while True:
            c = dict(kind=kind, V=_log(rng, 500, 131072), m=_log(rng, 128, 8192), t=_log(rng, 1, 8192), x=x)
            if rng.random() < 0.5:
                c.update(m=max(128, c["m"] // 128 * 128))
            if c["V"] * c["m"] * c["t"] <= 32000 * 4096 * 2048 and c["V"] * c["m"] <= 32000 * 8192:
                return c
    while True:
        c = dict(kind=kind, layers=rng.randint(1, 6), width=_log(rng, 33, 8192), inner=_log(rng, 64, 28672), x=rng.choice(["f16", "bf16", "f32"]),
                 limit=rng.choice([1.0, 1.0, 1e4]))
        if work(c)["bytes"] <= 1.6e9:
            return c


# ---- inputs -----------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _channels(m, gen):
    """Log-normal scale per channel, and outlier channels in runs."""
    scale = torch.exp(0.5 * _normal((m,), gen))
    first = torch.randint(0, max(1, m - RUN), (max(1, m // 800),), generator=gen, device="cuda")
    scale[(first[:, None] + torch.arange(RUN, device="cuda")).reshape(-1).clamp_(max=m - 1)] *= 50.0
    return scale


def _activations(t, m, dtype, gen):
    return (_normal((t, m), gen) * _channels(m, gen)).clamp_(-65504.0, 65504.0).to(dtype)


def _gradients(t, n, dtype, gen):
    """Gradients of outputs: tokens of very different weight, some of none (padding)."""
    g = _normal((t, n), gen) * torch.exp(1.5 * _normal((t, 1), gen)) * 1e-2
    if t > 8:
        g[torch.randperm(t, generator=gen, device="cuda")[: t // 8]] = 0.0
    return g.to(dtype)


def _stored(v, s_exp):
    """Numbers (already divided by their scales) and the exponents of the scales in the stored form: rows of e4m3 numbers padded with
    zeros to whole blocks, an odd number of them, rows of scale bytes padded to a multiple of four."""
    blocks = -(-v.shape[1] // BLOCK) | 1
    q = torch.zeros((v.shape[0], blocks * BLOCK), dtype=torch.uint8, device="cuda")
    q[:, : v.shape[1]] = v.to(E4M3).view(torch.uint8)
    s = torch.zeros((s_exp.shape[0], -(-s_exp.shape[1] // 4) * 4), dtype=torch.uint8, device="cuda")
    s[:, : s_exp.shape[1]] = (s_exp + 127).to(torch.uint8)
    return q.view(E4M3)[:, : v.shape[1]], s[:, : s_exp.shape[1]]


def _weights(n, m, gen):
    """A layer's weights in the stored form, and the same transposed: the blocks are square, so both hold the same numbers."""
    nb, mb = -(-n // BLOCK), -(-m // BLOCK)
    W = torch.zeros((nb * BLOCK, mb * BLOCK), device="cuda")
    W[:n, :m] = 0.02 * _normal((n, m), gen) * _channels(m, gen).clamp_(max=8.0)
    tiles = W.view(nb, BLOCK, mb, BLOCK)
    e = _exponents(tiles.abs().amax(dim=(1, 3)))
    scaled = (tiles * torch.exp2(-e)[:, None, :, None]).view(nb * BLOCK, mb * BLOCK)[:n, :m]
    return _stored(scaled, e) + _stored(scaled.t(), e.t())


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    s = dict(case=case, kind=kind)
    if kind in ("add_norm", "add_norm_grad"):
        rows, cols, x, w = case["rows"], case["cols"], DTYPES[case["x"]], DTYPES[case["w"]]
        s["X"] = (0.3 * _activations(rows, cols, torch.float32, gen)).to(x)                     # what the branch gave
        s["R"] = (_activations(rows, cols, torch.float32, gen) + 0.2 * _normal((1, cols), gen)).to(x)
        s["w"] = (1.0 + 0.3 * _normal((cols,), gen)).to(w)
        s["b"] = (0.1 * _normal((cols,), gen)).to(w) if case["bias"] else None
        if kind == "add_norm_grad":
            s["dY"], s["dH"] = _gradients(rows, cols, x, gen), _gradients(rows, cols, x, gen)
    elif kind in ("linear", "linear_grad"):
        n, m, t = case["n"], case["m"], case["t"]
        s["W"], s["Ws"], s["Wt"], s["Wts"] = _weights(n, m, gen)
        s["bias"] = s["res"] = None
        if kind == "linear":
            y = DTYPES[case["y"]]
            if case["x"] == "e4m3":
                s["Xq"], s["Xs"] = _stored(*_blocks(_activations(t, m, torch.float32, gen)))
            else:
                s["X"] = _activations(t, m, DTYPES[case["x"]], gen)
            if case["bias"]:
                s["bias"] = _normal((n,), gen).to(y)
            if case["res"]:
                s["res"] = (3.0 * _normal((t, n), gen)).to(y)
        else:
            x = DTYPES[case["x"]]
            s["X"] = _activations(t, m, x, gen)
            s["dY"] = _gradients(t, n, x, gen)
            s["Z"] = (1.5 * _normal((t, n), gen)).to(x) if case["act"] != "none" else None
    elif kind in ("head", "head_grad"):
        V, m, t, x = case["V"], case["m"], case["t"], DTYPES[case["x"]]
        s["W"], s["Ws"], s["Wt"], s["Wts"] = _weights(V, m, gen)
        s["labels"] = torch.randint(0, V, (t,), generator=gen, device="cuda")
        # hidden states behind a norm; many of them know their label a little
        known = torch.rand((t, 1), generator=gen, device="cuda") * 6.0
        toward = _dequantised(s["W"].view(torch.uint8)[s["labels"]].view(E4M3), s["Ws"][s["labels"] // BLOCK], 1)
        toward = toward / toward.square().sum(dim=1, keepdim=True).sqrt().clamp(min=1e-6)
        s["X"] = (_normal((t, m), gen) + known * toward).to(x)
        if t > 8:                                                   # padding
            s["labels"][torch.randperm(t, generator=gen, device="cuda")[: t // 8]] = -100
        s["dloss"] = torch.full((t,), 1.0 / t, device="cuda")
    else:
        x, w, i = DTYPES[case["x"]], case["width"], case["inner"]
        shapes = ([(w, w)] * 4 + [(i, w)] * 3 + [(w,)] * 2) * case["layers"]
        total = math.sqrt(sum(math.prod(v) for v in shapes))
        # per-tensor weight; the norm of all is between 1 and 10, say.  Vectors are the norms' gradients, in fp32
        s["g"] = [(_normal(v, gen) * torch.exp(_normal((1,), gen)) * (2.0 / total)).to(x if len(v) == 2 else torch.float32) for v in shapes]
        s["out"] = [torch.empty_like(v) for v in s["g"]]
    return s


# ---- the plain form -----------------------------------------------------------------------------------------------
def _exponents(a):
    """The exponent of the scale of blocks whose largest magnitude is a."""
    f, e = torch.frexp(a)                                   # a = f 2^e, f in [1/2, 1);  448 = 7/8 2^9
    e = (e - 9 + (f > 0.875)).clamp_(min=-126)
    return torch.where(a > 0, e, -126).float()


def _blocks(x):
    """x (rows x cols, fp32) in blocks of 128 along its rows: the numbers over their scales, and the scales' exponents."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x, (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    e = _exponents(torch.where(torch.isfinite(v), v.abs(), 0.0).amax(dim=2))
    v = torch.where(torch.isfinite(v), v / torch.exp2(e)[:, :, None], math.nan)
    return v.view(rows, -1)[:, :cols], e


def _quantised(x):
    """Q(x) as fp32 numbers."""
    v, e = _blocks(x.float())
    return v.to(E4M3).float() * torch.exp2(e).repeat_interleave(BLOCK, 1)[:, : x.shape[1]]


def _dequantised(q, s, rows=BLOCK):
    """Stored numbers as fp32 numbers; `rows`: of a block."""
    n, m = q.shape
    s = torch.exp2(s.float() - 127.0)
    return q.float() * s.repeat_interleave(rows, 0)[:n].repeat_interleave(BLOCK, 1)[:, :m]


def _plain_norm(s, backward):
    c = s["case"]
    x = s["X"].dtype
    h = (s["X"].float() + s["R"].float()).to(x)
    v, w = h.float(), s["w"].float()
    d = v if c["rms"] else v - v.mean(dim=1, keepdim=True)
    r = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    hh = d * r
    y = hh * w
    if s["b"] is not None:
        y = y + s["b"].float()
    y = y.to(x)
    out = dict(h=h)
    if c["y"]:
        out["y"] = y
    if c["q"]:
        q, e = _blocks(y.float())
        out["q"], out["s"] = q.to(E4M3), (e + 127).to(torch.uint8).view(E8M0)
    if not backward:
        return out
    dy = s["dY"].float()
    g = dy * w
    dx = g - hh * (g * hh).mean(dim=1, keepdim=True)
    if not c["rms"]:
        dx = dx - g.mean(dim=1, keepdim=True)
    out.update(dx=(s["dH"].float() + dx * r).to(x), dw=(dy * hh).sum(dim=0).to(s["w"].dtype))
    if s["b"] is not None:
        out["db"] = dy.sum(dim=0).to(s["w"].dtype)
    return out


def _activated(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return z * 0.5 * torch.erfc(z * -math.sqrt(0.5))
    return z / (1.0 + torch.exp(-z)) if act == "silu" else z


def _slope(z, act):
    if act == "relu":
        return (z > 0.0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    sigma = 1.0 / (1.0 + torch.exp(-z))
    return sigma * (1.0 + z * (1.0 - sigma))


def _plain_linear(s):
    c = s["case"]
    y = DTYPES[c["y"]]
    x = _dequantised(s["Xq"], s["Xs"], 1) if c["x"] == "e4m3" else _quantised(s["X"])
    z = torch.mm(x, _dequantised(s["W"], s["Ws"]).t())
    if s["bias"] is not None:
        z = z + s["bias"].float()
    out = _activated(z, c["act"])
    if s["res"] is not None:
        out = out + s["res"].float()
    return dict(y=out.to(y), z=z.to(y)) if c["z"] else out.to(y)


def _plain_linear_grad(s):
    c, x = s["case"], s["X"].dtype
    dz = s["dY"].float()
    if c["act"] != "none":
        dz = dz * _slope(s["Z"].float(), c["act"])
    r = dz.to(x)
    out = dict(dx=torch.mm(_quantised(r), _dequantised(s["W"], s["Ws"])).to(x),
               dw=torch.mm(_quantised(r.t()), _quantised(s["X"].t()).t()).to(x))
    if c["bias"] != "none":
        out["db"] = dz.sum(dim=0).to(DTYPES[c["bias"]])
    return out


def _plain_head(s, backward):
    W, V = _dequantised(s["W"], s["Ws"]), s["W"].shape[0]
    x = _quantised(s["X"])
    z = torch.mm(x, W.t())
    top = z.amax(dim=1, keepdim=True).double()
    # (a sum of exponentials, and the difference of two large numbers that the loss is: in 64 bits)
    lse = top[:, 0] + torch.log(torch.exp(z.double() - top).sum(dim=1))
    live = (s["labels"] >= 0) & (s["labels"] < V)
    at = torch.where(live, s["labels"], 0)[:, None]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0].double(), 0.0).float()
    if not backward:
        return loss
    g = torch.where(live, s["dloss"], 0.0)[:, None]
    dz = torch.exp(z.double() - lse[:, None])
    dz = dz.scatter_add_(1, at, torch.full_like(dz[:, :1], -1.0)).float() * g
    return dict(loss=loss, dx=torch.mm(_quantised(dz), W).to(s["X"].dtype),
                dw=torch.mm(_quantised(dz.t()), _quantised(s["X"].t()).t()).to(s["X"].dtype))


def _plain_clip(s):
    norm = torch.stack([v.double().square().sum() for v in s["g"]]).sum().sqrt()
    factor = (s["case"]["limit"] / norm).clamp(max=1.0).float()
    return dict(norm=norm.float(), g=[(v.float() * factor).to(v.dtype) for v in s["g"]])


def _plain(s):
    kind = s["kind"]
    if kind in ("add_norm", "add_norm_grad"):
        return _plain_norm(s, kind == "add_norm_grad")
    if kind == "linear":
        return _plain_linear(s)
    if kind == "linear_grad":
        return _plain_linear_grad(s)
    if kind in ("head", "head_grad"):
        return _plain_head(s, kind == "head_grad")
    return _plain_clip(s)


# ---- the framework's operators ------------------------------------------------------------------------------------
_slim = None


def _context():
    """What a user's program keeps for all of its layers: one library context."""
    global _slim
    if _slim is None:
        from paper_2405_14917_amd import binding
        _slim = binding.Slim("cuda:0")
    return _slim


def _own(s):
    kind, c, slim = s["kind"], s["case"], _context()
    if kind in ("add_norm", "add_norm_grad"):
        grad = kind == "add_norm_grad"
        o = slim.add_norm(s["X"], s["R"], s["w"], s["b"], EPS, rms=c["rms"], y=c["y"], e4m3=c["q"], stats=grad)
        out = dict(h=o.H)
        if c["y"]:
            out["y"] = o.Y
        if c["q"]:
            out["q"], out["s"] = o.q, o.s.view(E8M0)
        if grad:
            dx, dw, db = slim.add_norm_backward(s["dY"], s["dH"], o.H, s["w"], o.mean, o.rstd, bias=c["bias"])
            out.update(dx=dx, dw=dw)
            if c["bias"]:
                out["db"] = db
        return out
    if kind == "linear":
        x = (s["Xq"], s["Xs"]) if c["x"] == "e4m3" else s["X"]
        out = slim.fp8_linear_act(x, s["W"], s["Ws"], s["bias"], c["act"], s["res"], dtype=DTYPES[c["y"]], keep=c["z"])
        return dict(y=out[0], z=out[1]) if c["z"] else out
    if kind == "linear_grad":
        dx, dw, db = slim.fp8_linear_act_backward(s["dY"], s["Z"], c["act"], s["X"], s["Wt"], s["Wts"], db_dtype=DTYPES.get(c["bias"]))
        return dict(dx=dx, dw=dw) if db is None else dict(dx=dx, dw=dw, db=db)
    if kind == "head":
        return slim.head_loss(s["X"], s["W"], s["Ws"], s["labels"])
    if kind == "head_grad":
        loss, dx, dw = slim.head_loss_grad(s["X"], s["W"], s["Ws"], s["Wt"], s["Wts"], s["labels"], s["dloss"])
        return dict(loss=loss, dx=dx, dw=dw)
    return dict(norm=slim.clip_gradients(s["g"], c["limit"], out=s["out"]), g=s["out"])


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ---- what the work cannot do without ------------------------------------------------------------------------------
def _size(name):
    return {"f32": 4.0, "e4m3": 1.0 + 1.0 / BLOCK, "none": 0.0}.get(name, 2.0)


def work(case):
    kind = case["kind"]
    if kind in ("add_norm", "add_norm_grad"):
        cells, cols, x, w = float(case["rows"] * case["cols"]), case["cols"], _size(case["x"]), _size(case["w"])
        k = 2.0 if case["bias"] else 1.0
        forward = cells * (3.0 * x + (x if case["y"] else 0.0) + (_size("e4m3") if case["q"] else 0.0)) + k * w * cols
        if kind == "add_norm":
            return dict(bytes=forward, flops=10.0 * cells)
        return dict(bytes=forward + 3.0 * x * cells + k * w * cols, flops=24.0 * cells)
    if kind in ("linear", "linear_grad"):
        n, m, t = case["n"], case["m"], case["t"]
        stored = n * m + float(-(-n // BLOCK)) * (-(-m // BLOCK))
        if kind == "linear":
            y = _size(case["y"])
            return dict(bytes=stored + _size(case["x"]) * t * m + y * n * t * (1 + case["res"] + case["z"]) + y * n * case["bias"], flops=2.0 * n * m * t)
        x = _size(case["x"])
        return dict(bytes=stored + x * (t * n * (1 + (case["act"] != "none")) + 2.0 * t * m + float(n) * m) + _size(case["bias"]) * n, flops=4.0 * n * m * t)
    if kind in ("head", "head_grad"):
        V, m, t = case["V"], case["m"], case["t"]
        stored = V * m + float(-(-V // BLOCK)) * (-(-m // BLOCK))
        if kind == "head":
            return dict(bytes=stored + 2.0 * t * m + 12.0 * t, flops=2.0 * V * m * t)
        return dict(bytes=stored + 4.0 * t * m + 2.0 * V * m + 16.0 * t, flops=6.0 * V * m * t)      # (either form holds the weights)
    w, i, x = float(case["width"]), float(case["inner"]), _size(case["x"])
    cells, vectors = case["layers"] * (4 * w * w + 3 * i * w), case["layers"] * 2 * w
    return dict(bytes=2.0 * (x * cells + 4.0 * vectors) + 4.0, flops=3.0 * (cells + vectors))


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------
def _exact_e4m3(v):
    """The e4m3 number nearest to v, |v| <= 448 + half a step: three binary digits behind the first one, none below 2^-9."""
    digit = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -30)))
    digit = digit + (torch.exp2(digit + 1) <= v.abs()).double() - (torch.exp2(digit) > v.abs()).double()
    step = torch.exp2(torch.clamp(digit, min=-6.0) - 3.0)
    return torch.round(v / step) * step                    # (round: ties to even)


def _exact_blocks(x):
    """(e4m3 numbers, scales) of blocks of 128 along the rows of x."""
    x = x.double()
    q, scales = torch.empty_like(x), []
    for b in range(0, x.shape[1], BLOCK):
        v = x[:, b: b + BLOCK]
        a = v.abs().amax(dim=1, keepdim=True)
        s = torch.exp2(torch.ceil(torch.log2((a / 448.0).clamp(min=2.0 ** -140))).clamp(min=-126.0))
        s = torch.where(a > 448.0 * s, 2.0 * s, torch.where((a <= 224.0 * s) & (s > 2.0 ** -126), 0.5 * s, s))
        q[:, b: b + BLOCK] = _exact_e4m3(v / s)
        scales.append(s)
    return q, torch.cat(scales, dim=1)


def _exact_quantised(x):
    q, s = _exact_blocks(x)
    return q * s[:, torch.arange(x.shape[1], device=x.device) // BLOCK]


def _exact_weights(q, s, rows=BLOCK):
    i = torch.arange(q.shape[0], device="cuda") // rows
    j = torch.arange(q.shape[1], device="cuda") // BLOCK
    return q.double() * torch.pow(2.0, s.double() - 127.0)[i][:, j]


def _exact_act(z, act):
    """The activation and its slope."""
    if act == "relu":
        return torch.where(z > 0.0, z, 0.0), torch.where(z > 0.0, 1.0, 0.0).double()
    if act == "gelu":
        below = torch.special.ndtr(z)
        return z * below, below + z * torch.exp(-z.square() / 2.0) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        sigma = torch.sigmoid(z)
        return z * sigma, sigma + z * sigma * torch.sigmoid(-z)
    return z, torch.ones_like(z)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("add_norm", "add_norm_grad"):
        n, x = case["cols"], s["X"].dtype
        h = (s["X"].double() + s["R"].double()).to(x).double()
        w = s["w"].double()
        mean = torch.zeros_like(h[:, :1]) if case["rms"] else h.sum(dim=1, keepdim=True) / n
        sd = torch.sqrt(((h - mean) ** 2).sum(dim=1, keepdim=True) / n + EPS)
        hh = (h - mean) / sd
        y = hh * w + (0.0 if s["b"] is None else s["b"].double())
        out = dict(h=h)
        if case["y"]:
            out["y"] = y
        if case["q"]:
            out["q"], out["s"] = _exact_blocks(y.to(x))
        if kind == "add_norm":
            return out
        dy = s["dY"].double()
        dhh = dy * w                                        # through hh(h): the derivative of a row's projection
        along = (dhh * hh).sum(dim=1, keepdim=True) / n
        flat = torch.zeros_like(along) if case["rms"] else dhh.sum(dim=1, keepdim=True) / n
        out.update(dx=s["dH"].double() + (dhh - flat - along * hh) / sd, dw=(dy * hh).sum(dim=0))
        if s["b"] is not None:
            out["db"] = dy.sum(dim=0)
        return out
    if kind == "linear":
        x = _exact_weights(s["Xq"], s["Xs"], 1) if case["x"] == "e4m3" else _exact_quantised(s["X"])
        z = x @ _exact_weights(s["W"], s["Ws"]).t().contiguous()
        if case["bias"]:
            z = z + s["bias"].double()
        y = _exact_act(z, case["act"])[0]
        if case["res"]:
            y = y + s["res"].double()
        return dict(y=y, z=z) if case["z"] else y
    if kind == "linear_grad":
        dz = s["dY"].double()
        if case["act"] != "none":
            dz = dz * _exact_act(s["Z"].double(), case["act"])[1]
        r, xt = dz.to(s["dY"].dtype), s["X"].t().contiguous()
        out = dict(dx=_exact_quantised(r) @ _exact_weights(s["W"], s["Ws"]),
                   dw=_exact_quantised(r.t().contiguous()) @ _exact_quantised(xt).t().contiguous())
        if case["bias"] != "none":
            out["db"] = dz.sum(dim=0)
        return out
    if kind in ("head", "head_grad"):
        W, V = _exact_weights(s["W"], s["Ws"]), case["V"]
        z = _exact_quantised(s["X"]) @ W.t().contiguous()
        lnp = torch.log_softmax(z, dim=1)
        del z
        one = torch.zeros_like(lnp)
        live = (s["labels"] >= 0) & (s["labels"] < V)
        one[torch.nonzero(live)[:, 0], s["labels"][live]] = 1.0
        loss = -torch.where(one > 0.0, lnp, 0.0).sum(dim=1)
        if kind == "head":
            return loss
        dz = (torch.exp(lnp) - one) * torch.where(live, s["dloss"].double(), 0.0)[:, None]
        del lnp, one
        return dict(loss=loss, dx=_exact_quantised(dz) @ W,
                    dw=_exact_quantised(dz.t().contiguous()) @ _exact_quantised(s["X"].t().contiguous()).t().contiguous())
    squares = [float((v.double() ** 2).sum()) for v in s["g"]]
    norm = math.sqrt(math.fsum(squares))
    factor = 1.0 if norm <= case["limit"] else case["limit"] / norm
    return dict(norm=torch.tensor(norm, dtype=torch.float64), g=[v.double() * factor for v in s["g"]])

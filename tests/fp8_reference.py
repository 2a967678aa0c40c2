"""The 8-bit linear layer's definition in 64 bits, on the CPU."""
import torch

B = 128


def e4m3(v):
    """The e4m3 number nearest to |v| <= 448 (ties to even)."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -40)))
    e = e + (2.0 ** (e + 1) <= v.abs()).double() - (2.0 ** e > v.abs()).double()
    step = 2.0 ** (e.clamp(min=-6.0) - 3.0)
    return torch.round(v / step) * step


def exponent(a):
    """log2 of the smallest power of two s >= 2^-126 with a <= 448 s."""
    e = torch.ceil(torch.log2((a / 448.0).clamp(min=2.0 ** -200))).clamp(min=-126.0)
    e = torch.where(a > 448.0 * 2.0 ** e, e + 1, e)
    return torch.where((a <= 448.0 * 2.0 ** (e - 1)) & (e > -126), e - 1, e)


def quantize(x, rb=1, cb=B):
    """x in blocks of rb x cb: (stored numbers, exponents of the scales, their product)."""
    x = x.double()
    rows, cols = x.shape
    nb, mb = -(-rows // rb), -(-cols // cb)
    v = torch.zeros((nb * rb, mb * cb), dtype=torch.float64)
    v[:rows, :cols] = x
    v = v.view(nb, rb, mb, cb)
    fine = torch.isfinite(v)
    a = torch.where(fine, v.abs(), 0.0).amax(dim=(1, 3))
    e = exponent(a)
    s = (2.0 ** e)[:, None, :, None]
    q = torch.where(fine, e4m3(torch.where(fine, v, 0.0) / s), float("nan"))
    full = lambda t: t.reshape(nb * rb, mb * cb)[:rows, :cols]
    return full(q), e, full(q * s)


def q_rows(x):
    return quantize(x)[2]


def q_cols(x):
    """x in blocks of 128 rows."""
    return quantize(x, B, 1)[2]

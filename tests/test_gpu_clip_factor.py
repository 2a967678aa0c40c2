"""The factor that gradients are scaled by, limit / norm, over the whole range of both: it may be far below what fp32 holds where the scaled gradients are ordinary
numbers.

The sum of squares and the factor are taken in fp64 (2^-40 covers them), the product too; it is rounded to fp32 and, where its type has 16 bits, from there once
more: half a step of each, at least half of the type's smallest number."""
import pytest
import torch

from test_gpu_clip import HALF, U, exact_norm

pytestmark = pytest.mark.gpu

LEAST = {torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}


@pytest.fixture(scope="module")
def slim():
    from paper_2405_14917_amd import binding
    s = binding.Slim("cuda:0")
    yield s
    s.close()


@pytest.mark.parametrize("big,limit", [(3e37, 1.0), (3e37, 1e-3), (3e37, 1e-6), (1e38, 1e-7), (1e38, 1e-30), (3e4, 1e-6), (1.0, 1e-3), (1.0, 0.7), (1e-30, 1e-34)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_scaled_to_half_a_step(slim, big, limit, dtype):
    g = torch.Generator().manual_seed(3)
    one = torch.tensor([big, -big, big / 3, big * 2.0 ** -9]).to(dtype if big < 6e4 else torch.bfloat16).cuda()
    wide = torch.zeros((3, 9), dtype=dtype, device="cuda")
    wide[:, 2:7] = (torch.randn((3, 5), generator=g) * min(big, 1e4) * 0.1).to(dtype).cuda()
    tensors = [one, wide[:, 2:7], (torch.randn(5000, generator=g) * min(big, 1e4) * 0.01).to(dtype).cuda()]
    want = exact_norm(tensors)
    keep = [t.clone() for t in tensors]
    n = slim.clip_gradients(tensors, limit)
    assert abs(float(n) - want) <= (U + 2.0 ** -40) * want
    for t, k in zip(tensors, keep):
        f = k.double() * (limit / want if want > limit else 1.0)
        steps = HALF[t.dtype] + (U if t.dtype != torch.float32 else 0.0) + 2.0 ** -40
        assert bool(((t.double() - f).abs() <= steps * f.abs() + 0.51 * LEAST[t.dtype]).all()), float(((t.double() - f).abs() / f.abs().clamp(min=1e-300)).max())
    if limit < want:
        # (the sum of the scaled squares is the limit's, as far as these roundings go, unless they fall below the type's smallest numbers)
        assert limit < 1e-3 or abs(exact_norm(tensors) - limit) <= (HALF[dtype] + HALF[torch.bfloat16]) * limit
    assert not wide[:, :2].any() and not wide[:, 7:].any()

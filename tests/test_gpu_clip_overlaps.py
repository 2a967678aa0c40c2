"""Outputs of the scaling of gradients that lie in other tensors' memory are refused, with nothing written; those side by side in one matrix are not."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_outputs_in_other_tensors_places():
    from paper_2405_14917_amd import binding
    slim = binding.Slim("cuda:0")
    a, b, wide = torch.randn((300, 70), device="cuda"), torch.randn((300, 70), device="cuda"), torch.randn((300, 141), device="cuda")
    keep = [v.clone() for v in (a, b, wide)]
    norm = float(torch.sqrt((a.double() ** 2).sum() + (b.double() ** 2).sum()))
    for tensors, out in (([a, b], [b, a]), ([a, b], [torch.empty_like(a), a]), ([wide[:, :70]], [wide[:, 1:71]]), ([wide[:, :70], wide[:, 70:140]], [wide[:, 70:140], wide[:, :70]]),
                         ([wide[:, :70], wide[:, 69:139]], None), ([wide.view(-1)[70:], wide[:1, :71]], None)):
        with pytest.raises(binding.SlimError) as e:
            slim.clip_gradients(tensors, 0.1, out=out)
        assert e.value.status == binding.ERR_INVALID_ARG and "overlap" in str(e.value)
    assert all(torch.equal(v, k) for v, k in zip((a, b, wide), keep))
    n = slim.clip_gradients([a, b], 0.5, out=[wide[:, :70], wide[:, 71:]])
    assert abs(float(n) - norm) <= 2.0 ** -23 * norm
    for got, k in ((wide[:, :70], keep[0]), (wide[:, 71:], keep[1])):
        f = k.double() * (0.5 / norm)
        assert bool(((got.double() - f).abs() <= 2.0 ** -22 * f.abs()).all())
    assert torch.equal(wide[:, 70], keep[2][:, 70])
    slim.clip_gradients([wide[:, :70], wide[:, 71:]], 1e9, out=[wide[:, :70], wide[:, 71:]])
    slim.close()

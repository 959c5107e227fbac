"""Matrices without elements have a pitch whatever their strides say: a copy of one, which torch does not make, would not change them."""
import pytest
import torch

from paper_2511_12653_amd import binding as fq


@pytest.mark.parametrize("shape", [(0, 64), (5, 0), (0, 0), (0, 1)])
def test_pitch_of_nothing(shape):
    for t in (torch.zeros(shape), torch.zeros(1).expand(shape), torch.zeros(1).expand(shape).contiguous(), torch.zeros(shape[::-1]).t()):
        assert fq._pitch(t) == shape[1]


def test_other_pitches_are_checked():
    assert fq._pitch(torch.zeros(3, 8)[:, :5]) == 8
    for bad in (torch.zeros(8, 3).t(), torch.zeros(1, 8).expand(3, 8), torch.zeros(1).expand(3, 8)):
        with pytest.raises(ValueError):
            fq._pitch(bad)


@pytest.mark.gpu
def test_a_batch_of_nothing_trains_and_serves():
    from paper_2511_12653_amd import add_adapters, dropout, layer_norm, layer_norm_int8, linear_int8
    none = torch.zeros(1, device="cuda").expand(0, 64)
    for x in (torch.zeros(0, 64, device="cuda"), none, torch.zeros(2, 0, 64, device="cuda"), torch.zeros(1, device="cuda").expand(2, 0, 64)):
        x = x.detach().requires_grad_()
        w, b = torch.ones(64, device="cuda").requires_grad_(), torch.ones(64, device="cuda").requires_grad_()
        y = dropout(layer_norm(x, w, b), 0.1, 1, residual=x)
        gx, gw, gb = torch.autograd.grad(y.sum(), (x, w, b))              # (whose own gradient is one number, expanded)
        assert gx.shape == x.shape and not gw.any() and not gb.any()
        codes, scales = layer_norm_int8(x.detach(), w.detach(), b.detach())
        assert codes.shape == x.shape and scales.shape == x.shape[:-1]
    half = none.half()
    q, s = torch.zeros(48, 64, dtype=torch.int8, device="cuda"), torch.ones(48, device="cuda")
    base = linear_int8(half, q, s)
    a, b = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda"), torch.zeros(2, 48, 4, dtype=torch.float16, device="cuda")
    ids = torch.zeros(0, dtype=torch.int32, device="cuda")
    for given in (base, torch.zeros(1, dtype=torch.float16, device="cuda").expand(0, 48)):
        assert add_adapters(given, half, ids, a, b).shape == (0, 48)

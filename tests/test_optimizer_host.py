"""What the AdamW optimizer refuses before anything reaches a GPU: host logic, with tensors on the CPU that say they are on a card."""
import contextlib

import pytest
import torch

from paper_2511_12653_amd import AdamW
from paper_2511_12653_amd import binding as fq


class OnCard(torch.Tensor):
    """A tensor whose memory is the CPU's and whose device is card `card`."""
    card = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.card))

    def get_device(self):
        return self.card


def on_card(t, card=0, parameter=False):
    t = t.as_subclass(OnCard)
    t.card = card
    return t.requires_grad_() if parameter else t


def parameter(n=8, card=0, dtype=torch.float32):
    return on_card(torch.zeros(n, dtype=dtype), card, True)


@pytest.fixture
def no_gpu(monkeypatch):
    """Fails where the library is called."""
    def called(*_):
        raise AssertionError("the library was called")
    monkeypatch.setattr(torch.cuda, "device", lambda *_: contextlib.nullcontext())
    for name in ("fq_adamw_create", "fq_adamw_workspace_bytes", "fq_adamw_step"):
        monkeypatch.setattr(fq, name, called)


def test_a_step_is_not_captured(monkeypatch, no_gpu):
    p = parameter()
    opt = AdamW([p])
    p.grad = torch.ones(8).as_subclass(OnCard)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(RuntimeError, match="captur"):
        opt.step()
    assert opt.param_groups[0]["step"] == 0 and not opt.state


def refused():
    return [(RuntimeError, {"params": [torch.zeros(8, requires_grad=True)]}),
            (TypeError, {"params": [parameter(dtype=torch.float64)]}),
            (ValueError, {"params": [parameter()], "states": "float4"}),
            (ValueError, {"params": [parameter()], "copies": []}),
            (ValueError, {"params": [parameter()], "lr": float("inf")}),
            (ValueError, {"params": [parameter()], "lr": float("nan")}),
            (ValueError, {"params": [parameter()], "betas": (1.0, 0.999)}),
            (ValueError, {"params": [parameter()], "betas": (0.9, -0.1)}),
            (ValueError, {"params": [parameter()], "betas": (0.9, float("nan"))}),
            (ValueError, {"params": [parameter()], "eps": -1e-8}),
            (ValueError, {"params": [parameter()], "eps": float("inf")}),
            (ValueError, {"params": [parameter()], "weight_decay": float("nan")})]


@pytest.mark.parametrize("which", range(len(refused())))
def test_a_refused_group_does_not_stay(which):
    error, group = refused()[which]
    opt = AdamW([parameter()])
    for _ in range(2):
        with pytest.raises(error):
            opt.add_param_group(group)
        assert len(opt.param_groups) == 1
    with pytest.raises(error):
        AdamW([group])
    opt.add_param_group({"params": [parameter()], "lr": 1e-2, "seed": 5})
    assert len(opt.param_groups) == 2 and opt.param_groups[1]["seed"] == 5 + (1 << 32) and opt.param_groups[1]["lr"] == 1e-2


def test_a_group_lies_on_one_card(no_gpu, monkeypatch):
    opt = AdamW([parameter(card=1)])
    for given in ({"params": [parameter(), parameter(card=1)]},
                  {"params": [parameter(), parameter()], "copies": [None, on_card(torch.zeros(8, dtype=torch.float16), 1)]}):
        with pytest.raises(ValueError, match="GPU"):
            opt.add_param_group(given)
    opt.add_param_group({"params": [parameter(), parameter()]})      # (another group's card is its own)
    opt.add_param_group({"params": []})


def test_the_gradients_scale_lies_on_the_groups_card(no_gpu, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    p = parameter()
    p.grad = on_card(torch.ones(8))
    opt = AdamW([p])
    with pytest.raises(ValueError, match="GPU"):
        opt.step(grad_scale=on_card(torch.ones(1), 1))
    assert opt.param_groups[0]["step"] == 0 and not opt.state


def f32(card=0):
    return [on_card(torch.zeros(8), card) for _ in range(4)]


def test_a_list_lies_on_one_card(monkeypatch):
    params = [fq.FqParam.from_torch(*f32()), fq.FqParam.from_torch(*f32(1))]
    with pytest.raises(ValueError, match="GPU"):
        fq.fq_adamw_create(params, (1 << 20, 4096), stream=0)
    with pytest.raises(ValueError, match="GPU"):
        fq.fq_adamw_create(params[:1], on_card(torch.zeros(4096, dtype=torch.uint8), 1), stream=0)
    with pytest.raises(ValueError, match="GPU"):
        fq.FqParam.from_torch(*f32()[:3], f32(1)[0])


def test_sparse_gradients_are_refused(no_gpu, monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, **kw: zeros(*a, **kw))
    p = on_card(zeros(4, 2), parameter=True)
    opt = AdamW([p])
    dense = zeros(4, 2)
    dense[1] = 1.0
    p.grad = dense.to_sparse()
    with pytest.raises(TypeError, match="dense"):
        opt.step()
    assert opt.param_groups[0]["step"] == 0 and not opt.state

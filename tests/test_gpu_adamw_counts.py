"""What the AdamW optimizer counts as a step: updates of a group, from a parameter's first gradient on."""
import math

import pytest
import torch

from paper_2511_12653_amd import AdamW

pytestmark = pytest.mark.gpu

LR = 1e-2


def first_update(g):
    """A first update in 64 bits from p = 0: (1 - beta1) g / (1 - beta1) over sqrt((1 - beta2) g^2 / (1 - beta2)) + eps."""
    return -LR * g / (math.sqrt(g * g) + 1e-8)


def near(p, want):
    # about ten roundings to binary32, and those of 1 - beta in binary32 (beta2: 1e-3 of 2^-24 each)
    assert p.numel() and bool(((p.detach().double() - want).abs() <= 32 * 2.0 ** -24 * abs(want)).all()), (p.max(), want)


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_steps_without_a_gradient_do_not_count(states):
    p = torch.nn.Parameter(torch.zeros(300, device="cuda"))
    opt = AdamW([p], lr=LR, weight_decay=0.0, states=states)
    for _ in range(1000):
        opt.step()
    assert opt.param_groups[0]["step"] == 0
    p.grad = torch.full((300,), 0.25, device="cuda")
    opt.step()
    near(p, first_update(0.25))
    assert opt.param_groups[0]["step"] == 1


def test_refused_steps_do_not_count():
    a, b = (torch.nn.Parameter(torch.zeros(300, device="cuda")) for _ in range(2))
    opt = AdamW([{"params": [a]}, {"params": [b]}], lr=LR, weight_decay=0.0)
    a.grad, wrong = torch.full((300,), 0.25, device="cuda"), torch.full((600,), 0.25, device="cuda")[::2]
    b.grad = wrong
    for _ in range(3):
        with pytest.raises(TypeError):
            opt.step()
    b.grad = wrong.contiguous()
    opt.param_groups[1]["betas"] = (0.9, 1.0)
    for _ in range(3):
        with pytest.raises((ValueError, RuntimeError)):
            opt.step()
    opt.param_groups[1]["betas"] = (0.9, 0.999)
    with pytest.raises(TypeError):
        opt.step(grad_scale=torch.ones(2, device="cuda"))
    # neither group has moved, the one in front of the wrong one neither
    assert [g["step"] for g in opt.param_groups] == [0, 0] and not a.detach().any() and not b.detach().any()
    opt.step()
    near(a, first_update(0.25))
    near(b, first_update(0.25))
    assert [g["step"] for g in opt.param_groups] == [1, 1]


def test_a_refused_step_leaves_no_state():
    """A parameter whose first gradient was refused begins with the one that is not."""
    a, b = (torch.nn.Parameter(torch.zeros(300, device="cuda")) for _ in range(2))
    opt = AdamW([a, b], lr=LR, weight_decay=0.0)
    a.grad = torch.full((300,), 0.25, device="cuda")
    opt.step()
    b.grad = torch.full((600,), 0.25, device="cuda")[::2]
    with pytest.raises(TypeError):
        opt.step()
    b.grad = None
    opt.step()
    b.grad = torch.full((300,), 0.25, device="cuda")
    opt.step()
    near(b, first_update(0.25))


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_a_first_gradient_that_comes_late(states):
    import copy
    early, late = (torch.nn.Parameter(torch.zeros(300, device="cuda")) for _ in range(2))
    opt = AdamW([early, late], lr=LR, weight_decay=0.0, states=states, seed=4)
    for _ in range(1000):
        early.grad = torch.full((300,), 0.25, device="cuda")
        opt.step()
    assert not late.detach().any()
    late.grad = torch.full((300,), 0.25, device="cuda")
    opt.step()
    near(late, first_update(0.25))
    assert opt.param_groups[0]["step"] == 1001
    # it goes on from there as one that began then, also from a saved state
    alone = torch.nn.Parameter(torch.zeros(300, device="cuda"))
    other = AdamW([alone], lr=LR, weight_decay=0.0, states=states, seed=4)
    alone.grad = late.grad.clone()
    other.step()
    assert torch.equal(alone, late)
    saved, value = copy.deepcopy(opt.state_dict()), late.detach().clone()
    late.grad = alone.grad = torch.full((300,), -0.5, device="cuda")
    opt.step()
    other.step()
    assert torch.equal(alone, late)
    again = AdamW([early, late], lr=LR, weight_decay=0.0, states=states, seed=4)
    again.load_state_dict(saved)
    with torch.no_grad():
        late.copy_(value)
    again.step()
    assert torch.equal(alone, late)

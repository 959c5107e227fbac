"""What linear_int8 and the AdamW optimizer write counts as written for autograd, and linear_int8 loses neither a tangent nor a
history."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2511_12653_amd import AdamW, linear_int8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_a_step_after_the_forward_is_seen_by_backward(states):
    p = torch.nn.Parameter(torch.randn(300, device="cuda"))
    with torch.inference_mode():
        quiet = torch.zeros(300, dtype=torch.float16, device="cuda")
    half = torch.zeros(300, dtype=torch.float16, device="cuda")
    q = torch.nn.Parameter(torch.randn(300, device="cuda"))
    opt = AdamW([{"params": [p, q], "copies": [half, quiet]}], states=states)
    for _ in range(2):                               # (with a new plan, and with one that is there)
        p.grad = q.grad = torch.ones(300, device="cuda")
        x = torch.ones(300, device="cuda", requires_grad=True)
        y = torch.ones(300, device="cuda", dtype=torch.float16, requires_grad=True)
        for loss in ((x * p).sum(), (y * half).sum()):
            opt.step()
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
    assert torch.equal(quiet, q.detach().half())


def operands():
    torch.manual_seed(1)
    return torch.randn(4, 16, device="cuda"), torch.ones(8, 16, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")


def test_a_given_output_counts_as_written():
    x, w, ws, b = operands()
    out = torch.ones(4, 8, device="cuda")
    loss = (torch.ones(4, 8, device="cuda", requires_grad=True) * out).sum()
    linear_int8(x, w, ws, b, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        assert torch.equal(linear_int8(x, w, ws, b, out=torch.ones(4, 8, device="cuda")), out)
        quiet = torch.ones(4, 8, device="cuda")
    assert torch.equal(linear_int8(x, w, ws, b, out=quiet), out)


@pytest.mark.parametrize("which", ["x", "w_scale", "bias", "x_scale"])
def test_linear_int8_refuses_a_tangent(which):
    x, w, ws, b = operands()
    given = {"x": x, "w": w, "w_scale": ws, "bias": b}
    if which == "x_scale":
        given.update(x=torch.ones(4, 16, dtype=torch.int8, device="cuda"), x_scale=torch.ones(4, device="cuda"))
    for grad in (True, False):
        with torch.set_grad_enabled(grad), forward_ad.dual_level():
            dual = dict(given)
            dual[which] = forward_ad.make_dual(given[which], torch.ones_like(given[which]))
            with pytest.raises(RuntimeError, match="gradient"):
                linear_int8(**dual)
            linear_int8(**given)                     # (a level alone is nothing)
    linear_int8(**given)


def test_linear_int8_refuses_an_output_with_a_history():
    x, w, ws, b = operands()
    out = torch.ones(4, 8, device="cuda", requires_grad=True) * 2
    with pytest.raises(RuntimeError, match="gradient"):
        linear_int8(x, w, ws, b, out=out)
    assert bool((out == 2).all())
    with torch.no_grad():
        linear_int8(x, w, ws, b, out=out)
    assert torch.equal(out.detach(), linear_int8(x, w, ws, b))


def test_linear_int8_in_a_function_transform():
    x, w, ws, b = operands()
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda t: linear_int8(t, w, ws, b), (x,), (torch.ones_like(x),))
    with pytest.raises(RuntimeError):
        torch.func.grad(lambda t: linear_int8(t, w, ws, b).sum())(x)

"""What linear_int8 and the AdamW optimizer write counts as written for autograd."""
import pytest
import torch

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

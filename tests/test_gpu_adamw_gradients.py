"""The AdamW optimizer keeps no gradient alive: after zero_grad() a gradient's memory is free, and a training loop needs one set."""
import weakref

import pytest
import torch

from paper_2511_12653_amd import AdamW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_gradients_die_with_zero_grad(states):
    torch.manual_seed(1)
    params = [torch.nn.Parameter(torch.randn(n, device="cuda")) for n in (1 << 20, 700, 1)]
    copy = torch.zeros(1 << 20, dtype=torch.float16, device="cuda")
    opt = AdamW([{"params": params, "copies": [copy, None, None]}], states=states)
    held = None
    for step in range(4):
        for p in params:
            p.grad = torch.randn(p.shape, device="cuda")
        watched = [weakref.ref(p.grad) for p in params]
        opt.step()
        opt.zero_grad()
        assert all(w() is None for w in watched), step
        if step:                                     # (the first one makes the states)
            assert held in (None, torch.cuda.memory_allocated())
            held = torch.cuda.memory_allocated()


def test_gradients_that_move_and_change_type():
    """New addresses, the same addresses for other gradients, and gradients of another type: what is stepped is what is there."""
    torch.manual_seed(2)
    start, grads = torch.randn(5000, device="cuda"), torch.randn(6, 5000, device="cuda")
    moved, fixed = (torch.nn.Parameter(start.clone()) for _ in range(2))
    opts = AdamW([moved], lr=1e-2), AdamW([fixed], lr=1e-2)
    fixed.grad = torch.empty(5000, device="cuda")
    kept = []
    for i, g in enumerate(grads):
        fixed.grad.copy_(g)
        moved.grad = g.clone()
        if i % 2:
            kept.append(moved.grad)                  # (the next one cannot have this one's address)
        for opt in opts:
            opt.step()
        moved.grad = None
        assert torch.equal(moved, fixed), i


def test_a_gradient_outlives_a_step_on_another_stream():
    """Its memory is not given away while another stream has yet to read it."""
    p = torch.nn.Parameter(torch.zeros(1 << 20, device="cuda"))
    opt = AdamW([p], lr=1e-2)
    big, side = torch.ones(8192, 8192, device="cuda"), torch.cuda.Stream()
    p.grad = torch.ones(1 << 20, device="cuda")
    at = p.grad.data_ptr()
    opt.step()                                       # (makes the plan, whose table may wait for the GPU)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        product = big
        for _ in range(20):                          # some 100 ms that the step has to wait for
            product = torch.mm(big, big, out=torch.empty_like(big))
        opt.step()
    p.grad = None
    assert torch.empty(1 << 20, device="cuda").data_ptr() != at
    assert not side.query()                          # (or this has shown nothing)
    torch.cuda.current_stream().wait_stream(side)
    assert bool((p.detach() < -1.9e-2).all())


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_half_gradients_of_float_parameters(states):
    """What torch refuses until grad_dtype allows it; the same bits as with the gradients' values in FP32."""
    torch.manual_seed(3)
    start, g = torch.randn(900, device="cuda"), torch.randn(900, device="cuda", dtype=torch.float16)
    ends = []
    for dtype in (torch.float32, torch.float16):
        p = torch.nn.Parameter(start.clone())
        p.grad_dtype = dtype
        copy = torch.zeros(900, device="cuda", dtype=torch.float16)
        opt = AdamW([{"params": [p], "copies": [copy]}], lr=1e-2, states=states, seed=7)
        for _ in range(3):
            p.grad = g.to(dtype)
            opt.step()
        assert torch.equal(copy, p.detach().half())
        ends.append(p.detach())
    assert torch.equal(*ends)

"""The front doors' own float32 buffers (statistics of a norm, scales of codes, states of AdamW) are that whatever torch's default type is, which a program
that trains in float16 or checks in float64 sets."""
import pytest
import torch

from paper_2511_12653_amd import AdamW, add_adapters, dropout, fake_quantize, layer_norm, layer_norm_int8, linear_int8

pytestmark = pytest.mark.gpu


@pytest.fixture(params=[torch.float16, torch.bfloat16, torch.float64])
def other_default(request):
    torch.set_default_dtype(request.param)
    yield
    torch.set_default_dtype(torch.float32)


def rand(*shape, dtype=torch.float32, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.float32).to(dtype)


def train():
    x, w, b = rand(40, 72).requires_grad_(), rand(72, seed=1).requires_grad_(), rand(72, seed=2).requires_grad_()
    y = dropout(layer_norm(x, w, b), 0.1, 3, residual=x)
    return (y.detach(), *torch.autograd.grad(y, (x, w, b), rand(40, 72, seed=3)))


def serve():
    x = rand(40, 64, dtype=torch.float16)
    codes, scales = layer_norm_int8(x, rand(64, seed=1), rand(64, seed=2))
    q = (rand(48, 64, seed=4) * 40).clamp(-127, 127).to(torch.int8)
    y = linear_int8(codes, q, rand(48, seed=5).abs(), x_scale=scales)
    ids = torch.arange(40, device="cuda") % 3
    return codes, scales, add_adapters(y, codes, ids, rand(3, 8, 64, dtype=torch.float16, seed=6), rand(3, 48, 8, dtype=torch.float16, seed=7), x_scale=scales)


def step(states):
    p = rand(300).requires_grad_()
    theta = rand(1, seed=1).requires_grad_()
    fake_quantize(p, theta).backward(rand(300, seed=2))
    optimizer = AdamW([p, theta], lr=0.01, states=states)
    for _ in range(2):
        optimizer.step()
    return p.detach(), theta.detach(), *(optimizer.state[p][name] for name in sorted(optimizer.state[p]) if torch.is_tensor(optimizer.state[p][name]))


def same(work, *args):
    other = work(*args)
    torch.set_default_dtype(torch.float32)
    for s, t in zip(other, work(*args), strict=True):
        assert s.dtype == t.dtype and torch.equal(s.view(torch.uint8), t.view(torch.uint8))


def test_training(other_default):
    same(train)


def test_serving(other_default):
    same(serve)


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_steps(other_default, states):
    same(step, states)

"""layer_norm(), layer_norm_int8(), dropout() and add_adapters(): what they make of torch tensors, their gradients, what they refuse, and
all of them together as a network trains and serves with them."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import AdamW, add_adapters, binding as fq, dropout, fake_quantize, layer_norm, layer_norm_int8, linear_int8

import _more_operators_ref as R

pytestmark = pytest.mark.gpu
host = lambda t: t.detach().cpu().numpy()     # noqa: E731


def rand(*shape, dtype=torch.float32, seed=0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


# ---------------------------------------------------------------------------------------------------------- layer norm
def as_rows(x, width):
    return host(x).reshape(-1, width)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("lead", [(), (5,), (3, 7), (2, 0, 4)])
def test_layer_norm_shapes_strides_and_gradients(lead, dtype):
    width = 72
    w, b = (1 + 0.2 * rand(width, seed=1)).requires_grad_(), rand(width, seed=2).requires_grad_()
    values, g = rand(*lead, width, dtype=dtype, seed=3), rand(*lead, width, dtype=dtype, seed=4)
    wide = torch.full((*lead, 2 * width), 9.0, dtype=dtype, device="cuda")
    wide[..., 5:5 + width] = values
    turned = values.transpose(0, -1).contiguous().transpose(0, -1)
    first = None
    for x in (values.clone(), wide[..., 5:5 + width].detach(), turned):
        x.requires_grad_()
        y = layer_norm(x, w, b)
        assert y.shape == x.shape and y.dtype == dtype
        got = (y, *torch.autograd.grad(y, (x, w, b), g))
        if first is None:
            first = got
            y64, off, mean, rstd = R.norm(as_rows(x, width), host(w), host(b), 1e-5)
            R.check(as_rows(y, width), y64, off, dtype == torch.float16)
            want = R.norm_backward(as_rows(x, width), as_rows(g, width), host(w), mean.astype(np.float32), rstd.astype(np.float32))
            for name, t in zip(("gx", "gweight", "gbias"), got[1:]):
                value, off = want[name]
                R.check(host(t).reshape(value.shape), value, off, t.dtype == torch.float16, name)
        assert all(torch.equal(s, t) for s, t in zip(got, first))


def test_layer_norm_takes_what_is_given():
    x, w, b = rand(9, 40).requires_grad_(), rand(40, seed=1).requires_grad_(), rand(40, seed=2).requires_grad_()
    for weight, bias in ((None, None), (w, None), (None, b), (w, b)):
        y = layer_norm(x, weight, bias, out_dtype=torch.float16)
        assert y.dtype == torch.float16
        wanted = [t for t in (x, weight, bias) if t is not None]
        grads = torch.autograd.grad(y.float().sum(), wanted)              # (a gradient that is one number, expanded)
        assert all(g.dtype == t.dtype and g.shape == t.shape and bool(torch.isfinite(g).all()) for g, t in zip(grads, wanted))
    frozen = layer_norm(x.detach(), w, b)
    gw, = torch.autograd.grad(frozen, w, torch.ones_like(frozen))
    y = layer_norm(x, w, b)
    assert torch.equal(torch.autograd.grad(y, w, torch.ones_like(y))[0], gw)
    half = layer_norm(x.detach().half(), w.detach().half(), b.detach().half())
    assert half.dtype == torch.float16


def test_layer_norm_int8_is_what_linear_int8_takes():
    x, w, b = rand(2, 11, 96, dtype=torch.float16), rand(96, seed=1), rand(96, seed=2)
    codes, scales = layer_norm_int8(x, w, b)
    q, s, near = R.codes(as_rows(x, 96), host(w), host(b), 1e-5)
    sure = near > 127 * 2.0 ** -23
    assert codes.shape == x.shape and scales.shape == (2, 11) and np.array_equal(host(scales).reshape(-1), s)
    assert np.array_equal(as_rows(codes, 96)[sure], q[sure])
    weights = torch.randint(-127, 128, (24, 96), dtype=torch.int8, device="cuda")
    # the codes of the float32 norm, quantized by the linear layer itself, differ only where y's own rounding crosses a border
    y = linear_int8(codes, weights, torch.full((24,), 0.01, device="cuda"), x_scale=scales, out_dtype=torch.float32)
    z = linear_int8(layer_norm(x, w, b, out_dtype=torch.float32), weights, torch.full((24,), 0.01, device="cuda"))
    # a code may be off by one in one place of a thousand: 127 * scale * 0.01 then
    assert float((y - z).abs().max()) <= 4 * 127 * 0.01 * float(scales.max())


def test_layer_norm_refuses():
    x, w = rand(4, 16), rand(16)
    with pytest.raises(RuntimeError):
        layer_norm(x.cpu(), w)
    with pytest.raises(RuntimeError):
        layer_norm_int8(x.requires_grad_(), w)
    x = x.detach()
    for bad in (lambda: layer_norm(x, w[:8]), lambda: layer_norm(x, w, w.view(4, 4)), lambda: layer_norm(x, w.cpu()), lambda: layer_norm(x[0, 0])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: layer_norm(x.double()), lambda: layer_norm(x, w, w.half()), lambda: layer_norm(x, w, out_dtype=torch.float64)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(fq.FqError):
        layer_norm(x, w, eps=-1.0)
    y = layer_norm(x.requires_grad_(), w)
    gx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        gx.sum().backward()                                   # no second derivative, and no wrong one
    with pytest.raises(RuntimeError):
        y = layer_norm(x * 1.0, w)
        saved = layer_norm(x, w)
        with torch.no_grad():
            x.mul_(2.0)
        saved.sum().backward()                                # what it has saved has changed


# ------------------------------------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_dropout_and_its_gradients(dtype):
    x, r, g = rand(5, 33, 7, dtype=dtype, seed=1), rand(5, 33, 7, seed=2), rand(5, 33, 7, seed=3)
    for p in (0.0, 0.3, 1.0):
        for residual in (None, r):
            a = x.clone().requires_grad_()
            b = None if residual is None else residual.clone().requires_grad_()
            y = dropout(a, p, 17, 4, b)
            half = y.dtype == torch.float16
            assert y.dtype == (dtype if b is None else torch.float32)
            assert np.array_equal(host(y), R.dropout(host(x), p, 17, 4, None if b is None else host(r), half))
            grads = torch.autograd.grad(y, [a] if b is None else [a, b], g.to(y.dtype))
            assert np.array_equal(host(grads[0]), R.dropout(host(g.to(y.dtype)), p, 17, 4, None, dtype == torch.float16))
            assert b is None or torch.equal(grads[1], g)
    turned = x.transpose(0, 2).contiguous().transpose(0, 2).requires_grad_()       # places go by the tensor's order, not memory's
    assert torch.equal(dropout(turned, 0.3, 17, 4), dropout(x, 0.3, 17, 4))
    assert not torch.equal(dropout(x, 0.3, 17, 5), dropout(x, 0.3, 17, 4))
    both = x.float().requires_grad_()
    y = dropout(both, 0.3, 1, 0, both)
    gx, = torch.autograd.grad(y, both, g)
    assert np.array_equal(host(gx), host(g) + R.dropout(host(g), 0.3, 1, 0, None, False))


def test_dropout_step_on_the_gpu():
    x, step = rand(1000).requires_grad_(), torch.tensor([5], device="cuda")
    y = dropout(x, 0.5, 9, step)
    assert torch.equal(y, dropout(x, 0.5, 9, 5))
    y.sum().backward()
    y = dropout(x, 0.5, 9, step)
    step += 1
    with pytest.raises(RuntimeError):                         # the mask that the backward pass would make is another
        y.sum().backward()


def test_dropout_refuses():
    x = rand(4, 8)
    with pytest.raises(RuntimeError):
        dropout(x.cpu(), 0.1, 1)
    for bad in (lambda: dropout(x, 0.1, 1, residual=x[:2]), lambda: dropout(x, 0.1, -1), lambda: dropout(x, 0.1, 1, 1 << 64),
                lambda: dropout(x, 0.1, 1, torch.tensor([1]))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: dropout(x.double(), 0.1, 1), lambda: dropout(x, 0.1, 1, residual=x.half(), out_dtype=torch.float32),
                lambda: dropout(x, 0.1, 1, torch.tensor([1.0], device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(fq.FqError):
            dropout(x, p, 1)


# ------------------------------------------------------------------------------------------------------------ adapters
def adapter_operands(lead, k, n, count, rank, seed=0):
    base, x = rand(*lead, n, dtype=torch.float16, seed=seed), rand(*lead, k, dtype=torch.float16, seed=seed + 1)
    a = (rand(count, rank, k, seed=seed + 2) / k ** 0.5).half()
    b = (rand(count, n, rank, seed=seed + 3) / rank ** 0.5).half()
    ids = torch.randint(-1, count, lead, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    return base, x, ids, a, b


@pytest.mark.parametrize("lead", [(), (5,), (3, 30), (2, 0, 4)])
def test_add_adapters_shapes_and_strides(lead):
    base, x, ids, a, b = adapter_operands(lead, 64, 48, 3, 8)
    y = add_adapters(base, x, ids, a, b)
    want, off = R.adapters(host(x).reshape(-1, 64), None, host(ids).reshape(-1), host(a), host(b), None, host(base).reshape(-1, 48))
    R.check(host(y).reshape(-1, 48), want, off, True)
    wide = torch.zeros((*lead, 130), dtype=torch.float16, device="cuda")
    wide[..., 8:72] = x
    assert torch.equal(add_adapters(base, wide[..., 8:72], ids.int(), a, b), y)
    out = torch.empty_like(base)
    assert add_adapters(base, x, ids, a, b, out=out) is out and torch.equal(out, y)
    kept, before = base.clone(), base._version
    assert add_adapters(base, x, ids.to(torch.int16), a, b, out=base) is base and torch.equal(base, y) and base._version > before
    far = ids + (1 << 32)                                      # (none of the adapters, whatever its lower 32 bits say)
    assert torch.equal(add_adapters(kept, x, far, a, b), kept)
    assert add_adapters(kept, x, ids, a, b, torch.ones(3, device="cuda"), out_dtype=torch.float32).dtype == torch.float32


def test_add_adapters_refuses():
    base, x, ids, a, b = adapter_operands((6,), 64, 48, 3, 8)
    with pytest.raises(RuntimeError):
        add_adapters(base, x.cpu(), ids, a, b)
    with pytest.raises(RuntimeError):
        add_adapters(base, x, ids, a.clone().requires_grad_(), b)
    for bad in (lambda: add_adapters(base, x[:, :32], ids, a, b), lambda: add_adapters(base[:, :40], x, ids, a, b), lambda: add_adapters(base, x, ids[:5], a, b),
                lambda: add_adapters(base, x, ids, a[:2], b), lambda: add_adapters(base, x, ids, a, b, out=base[:5]), lambda: add_adapters(base, x, ids.cpu(), a, b),
                lambda: add_adapters(base, x, ids, a, b, torch.ones(2, device="cuda")), lambda: add_adapters(base, x.to(torch.int8), ids, a, b),
                lambda: add_adapters(base, x, ids, a.transpose(1, 2).contiguous().transpose(1, 2), b)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: add_adapters(base, x, ids.float(), a, b), lambda: add_adapters(base, x, ids, a.float(), b), lambda: add_adapters(base.double(), x, ids, a, b)):
        with pytest.raises(TypeError):
            bad()
    wide = torch.zeros(7, 48, dtype=torch.float16, device="cuda")
    with pytest.raises(fq.FqError):                            # the result would be written over what is still to be read
        add_adapters(wide[:6], x, ids, a, b, out=wide[1:])


# ------------------------------------------------------------------------------------------------------- all of them
class Block(torch.nn.Module):
    """h + dropout(linear(fake_quantize(layer_norm(h)))), and the same in int8 with adapters."""

    def __init__(self, width, seed):
        super().__init__()
        self.norm_w, self.norm_b = torch.nn.Parameter(torch.ones(width, device="cuda")), torch.nn.Parameter(torch.zeros(width, device="cuda"))
        self.weight = torch.nn.Parameter(rand(width, width, seed=seed) / width ** 0.5)
        self.theta_w = torch.nn.Parameter(torch.log(torch.expm1(self.weight.detach().abs().amax(1) / 127)))
        self.theta_x = torch.nn.Parameter(torch.log(torch.expm1(torch.full((1,), 4.0 / 127, device="cuda"))))
        self.seed = seed

    def forward(self, h, step, p=0.1, own=True):
        if own:
            x = layer_norm(h, self.norm_w, self.norm_b)
        else:
            x = (h - h.mean(-1, keepdim=True)) / (h.var(-1, correction=0, keepdim=True) + 1e-5).sqrt() * self.norm_w + self.norm_b
        y = fake_quantize(x, self.theta_x) @ fake_quantize(self.weight, self.theta_w, channel_dim=0).t()
        if own:
            return dropout(y, p, self.seed, step, residual=h)
        kept = torch.from_numpy(R.keep(y.numel(), p, self.seed, step)).cuda().view(y.shape)
        return h + torch.where(kept, y / (1 - p), 0.0)


def test_a_network_trains_and_serves_with_all_of_them():
    """Gradients of a step against those of the same network from torch's operations; ten steps of AdamW; then int8 with adapters."""
    width, tokens = 64, 96
    blocks = [Block(width, s) for s in (1, 2)]
    params = [q for m in blocks for q in m.parameters()]
    x, target = rand(tokens, width, seed=5), rand(tokens, width, seed=6)

    def loss(step, own):
        h = x
        for m in blocks:
            h = m(h, step, own=own)
        return (h - target).square().mean()

    a = torch.autograd.grad(loss(0, True), params)
    b = torch.autograd.grad(loss(0, False), params)
    for s, t in zip(a, b):
        # both in binary32, but a value next to the border of two codes may fall on either side: 1 of 127 steps of one value in a thousand
        assert float((s - t).norm()) <= 2e-2 * float(t.norm()) + 1e-6
    optimizer = AdamW(params, lr=1e-3, states="float8")
    before = [q.detach().clone() for q in params]
    for step in range(10):
        optimizer.zero_grad()
        value = loss(step, True)
        value.backward()
        optimizer.step()
        assert bool(torch.isfinite(value))
    assert all(not torch.equal(q, v) for q, v in zip(params, before))

    with torch.no_grad():
        ids = torch.randint(-1, 3, (tokens,), device="cuda")
        h = want = x
        for m in blocks:
            q, s = torch.empty(width, width, dtype=torch.int8, device="cuda"), torch.empty(width, device="cuda")
            fq.fq_forward(fq.FqTensor.from_torch(1, width, width, -127, 127, x=m.weight.detach().contiguous(), q=q, theta=m.theta_w.detach(), s=s))
            down = (rand(3, 8, width, seed=m.seed) / 8).half()
            up = (0.1 * rand(3, width, 8, seed=m.seed + 9)).half()
            codes, scales = layer_norm_int8(h, m.norm_w, m.norm_b)
            y = linear_int8(codes, q, s, x_scale=scales, out_dtype=torch.float32)
            h = dropout(add_adapters(y, codes, ids, down, up, x_scale=scales), 0.0, 0, residual=h)
            # the same in float64 torch: the codes stand for the norm up to half a code step (1 / 254 of a row's greatest)
            n = layer_norm(want, m.norm_w, m.norm_b).double()
            z = n @ (q.double() * s.double()[:, None]).t()
            for i in range(3):
                mine = (ids == i)[:, None]
                z = z + torch.where(mine, n @ down[i].double().t() @ up[i].double().t(), 0.0)
            want = (want.double() + z).float()
        assert float((h - want).norm() / want.norm()) < 3e-2


def test_on_another_stream_and_two_calls_at_once():
    """Calls on two streams at a time, each with memory of its own, give what they give alone."""
    x = [rand(3001, 384, dtype=torch.float16, seed=s) for s in (1, 2)]
    w, b = rand(384, seed=3).requires_grad_(), rand(384, seed=4).requires_grad_()
    base, _, ids, down, up = adapter_operands((3001,), 384, 256, 5, 16)

    def work(t):
        t = t.clone().requires_grad_()
        y = dropout(layer_norm(t, w, b), 0.2, 3)
        grads = torch.autograd.grad(y, (t, w, b), torch.ones_like(y))
        with torch.no_grad():
            return (y, *grads, add_adapters(base, y.detach(), ids, down, up))

    want = [work(t) for t in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for _ in range(5):
        got = []
        for t, stream in zip(x, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                got.append(work(t))
        for stream in streams:
            torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        for s, t in zip(got, want):
            assert all(torch.equal(u, v) for u, v in zip(s, t))


def test_captured_training_step():
    """Forward and backward passes in one graph, replayed with the program's own work between: every replay gives the eager result."""
    x, g = rand(500, 200), rand(500, 200, seed=1)
    w, b = rand(200, seed=2).requires_grad_(), rand(200, seed=3).requires_grad_()
    x.requires_grad_()
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def work():
        y = dropout(layer_norm(x, w, b), 0.1, 5, step, residual=x)
        return (y.detach(), *torch.autograd.grad(y, (x, w, b), g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = work()
    for turn in range(1, 5):
        with torch.no_grad():
            x.normal_()
            step.add_(turn)
        want = [t.clone() for t in work()]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(outs, want))

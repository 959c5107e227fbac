"""linear_int8() and the AdamW optimizer: what they make of torch tensors, against the plain implementation, what they refuse,
and the example that trains with the one and serves with the other."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2511_12653_amd import AdamW, linear_int8

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu


def operands(n, k, seed):
    rng = np.random.Generator(np.random.Philox(seed))
    w, ws, b = rng.integers(-127, 128, (n, k)).astype(np.int8), rng.uniform(1e-3, 2e-3, n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    return rng, w, ws, b


@pytest.mark.parametrize("lead", [(), (5,), (3, 7), (2, 0, 4)])
def test_linear_int8_shapes_and_strides(lead):
    rng, w, ws, b = operands(48, 96, 1)
    x = torch.randn((*lead, 96), device="cuda", dtype=torch.float16)
    wd, wsd, bd = H.dev(w), H.dev(ws), H.dev(b)
    q, s = R.quantize_rows(x.reshape(-1, 96).cpu().numpy())
    y, off = R.linear(q, s, w, ws, b, True)
    got = linear_int8(x, wd, wsd, bd)
    assert got.shape == (*lead, 48) and got.dtype == torch.float16
    R.check_linear(got.reshape(-1, 48).cpu().numpy(), y, off, True)
    # rows with gaps, rows of a transposed tensor, weights with a pitch, a given output
    wide = torch.zeros((*lead, 130), device="cuda", dtype=torch.float16)
    wide[..., 10:106] = x
    assert torch.equal(linear_int8(wide[..., 10:106], wd, wsd, bd), got)
    turned = x.unsqueeze(-1).transpose(-1, -2).squeeze(-2) if not lead else x.transpose(0, -1).contiguous().transpose(0, -1)
    assert torch.equal(linear_int8(turned, wd, wsd, bd), got)
    pitched = torch.zeros((48, 130), dtype=torch.int8, device="cuda")
    pitched[:, 3:99] = wd
    out = torch.zeros((*lead, 48), device="cuda", dtype=torch.float16)
    assert linear_int8(x, pitched[:, 3:99], wsd, bd, out=out) is out and torch.equal(out, got)
    codes = H.dev(q.astype(np.int8)).view(*lead, 96)
    if codes.numel():
        assert torch.equal(linear_int8(codes, wd, wsd, bd, x_scale=H.dev(s)), got)
        assert linear_int8(codes, wd, wsd, x_scale=H.dev(s[:1]), out_dtype=torch.float32).dtype == torch.float32


@pytest.mark.parametrize("rows", [3, 40])
def test_linear_int8_of_an_expanded_tensor(rows):
    _, w, ws, b = operands(48, 96, 4)
    x = torch.randn(1, 96, device="cuda")
    got = linear_int8(x.expand(rows, 96), H.dev(w), H.dev(ws), H.dev(b))
    assert torch.equal(got, linear_int8(x, H.dev(w), H.dev(ws), H.dev(b)).expand(rows, 48))


def test_linear_int8_refuses():
    _, w, ws, b = operands(8, 16, 2)
    x, wd, wsd, bd = torch.randn(4, 16, device="cuda"), H.dev(w), H.dev(ws), H.dev(b)
    with pytest.raises(RuntimeError):
        linear_int8(x.cpu(), wd, wsd)
    with pytest.raises(RuntimeError):
        linear_int8(x.requires_grad_(), wd, wsd)
    x = x.detach()
    for bad in (lambda: linear_int8(x[:, :8], wd, wsd), lambda: linear_int8(x, wd, wsd[:3]), lambda: linear_int8(x, wd, wsd, bd[:1]),
                lambda: linear_int8(x, wd, wsd, x_scale=torch.ones(4, device="cuda")), lambda: linear_int8(x.to(torch.int8), wd, wsd),
                lambda: linear_int8(x, wd, wsd, out=torch.zeros(4, 9, device="cuda")), lambda: linear_int8(x, wd.cpu(), wsd)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: linear_int8(x.double(), wd, wsd), lambda: linear_int8(x, wd.float(), wsd), lambda: linear_int8(x, wd, wsd.half())):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_adamw_steps_groups_and_restarts(states):
    """Groups with their own rate and decay, gradients that come and go, new gradient tensors every step, FP16 copies; and a
    second optimizer that goes on from the first one's state gives the same bits."""
    torch.manual_seed(3)
    make = lambda *s, **kw: torch.randn(*s, device="cuda", **kw)      # noqa: E731
    a, b, c = (torch.nn.Parameter(t) for t in (make(300, 7), make(11), make(513, dtype=torch.float16)))
    copy = torch.zeros(300, 7, device="cuda", dtype=torch.float16)
    groups = [{"params": [a, b], "weight_decay": 0.1, "copies": [copy, None]}, {"params": [c], "lr": 1e-2, "weight_decay": 0.0}]
    opt = AdamW(groups, lr=3e-3, states=states, seed=11)
    scale = torch.full((1,), 0.5, device="cuda")

    def grads(step):
        torch.manual_seed(100 + step)
        a.grad, b.grad, c.grad = make(300, 7), (make(11) if step != 2 else None), make(513, dtype=torch.float16)

    def states_of(p):
        s = opt.state[p]
        if not s:
            z = np.zeros(p.numel(), np.float32)
            blocks = np.zeros(-(-p.numel() // 256), np.float32)
            return z, z, *((blocks, blocks) if states == "float8" else (None, None))
        host = lambda t: None if t is None else t.float().cpu().numpy().reshape(-1)      # noqa: E731
        return host(s["m"]), host(s["v"]), host(s.get("m_scale")), host(s.get("v_scale"))

    for step in range(1, 5):
        grads(step)
        want = []
        for g, (params, lr, decay) in enumerate((([a, b], 3e-3, 0.1), ([c], 1e-2, 0.0))):
            place = 0
            h = dict(lr=lr, beta1=0.9, beta2=0.999, eps=1e-8, step=step, seed=11 + (g << 32))
            for p in params:
                if p.grad is None:
                    continue
                m, v, ms, vs = states_of(p)
                want.append((p, R.step(p.detach().cpu().numpy().reshape(-1), p.grad.cpu().numpy().reshape(-1), m, v, ms, vs, h, place,
                                       1.0, decay, np.float32(0.5))))
                place += -(-p.numel() // 256) * 256
        untouched = b.detach().clone()
        opt.step(grad_scale=scale)
        for p, w in want:
            far = np.abs(p.detach().cpu().numpy().reshape(-1).astype(np.float64) - w["p"]) - w["off"]
            assert far.max() <= 0, (step, tuple(p.shape))
            if states == "float32":
                assert np.array_equal(opt.state[p]["m"].cpu().numpy().reshape(-1), w["m"])
            else:
                assert np.array_equal(opt.state[p]["m"].float().cpu().numpy().reshape(-1), w["m8"].astype(np.float32))
        assert torch.equal(copy, a.detach().half())
        if step == 2:
            assert torch.equal(b, untouched)
    assert opt.param_groups[0]["step"] == 4

    saved = {k: v for k, v in opt.state_dict().items()}
    values = [p.detach().clone() for p in (a, b, c)]
    state = {"state": {i: {k: t.clone() for k, t in s.items()} for i, s in saved["state"].items()}, "param_groups": saved["param_groups"]}
    import copy as copying
    state = copying.deepcopy(state)
    grads(5)
    opt.step()
    ends = [p.detach().clone() for p in (a, b, c)]
    with torch.no_grad():
        for p, v in zip((a, b, c), values):
            p.copy_(v)
    again = AdamW([{"params": [a, b], "weight_decay": 0.1}, {"params": [c], "lr": 1e-2, "weight_decay": 0.0}], lr=3e-3, states=states, seed=11)
    again.load_state_dict(state)
    grads(5)
    again.step()
    for p, v in zip((a, b, c), ends):
        assert torch.equal(p, v)
    torch.optim.lr_scheduler.StepLR(again, 1)


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_adamw_copies_stay_the_programs_own(states):
    """A state that is loaded brings no copies with it and takes none away; an optimizer that was copied steps on its own."""
    import copy as copying
    torch.manual_seed(5)
    p = torch.nn.Parameter(torch.randn(700, device="cuda"))
    half = torch.zeros(700, device="cuda", dtype=torch.float16)
    opt = AdamW([{"params": [p], "copies": [half]}], lr=1e-2, states=states)
    p.grad = torch.randn(700, device="cuda")
    opt.step()
    saved = copying.deepcopy(opt.state_dict())
    assert all(g["copies"] is None for g in saved["param_groups"])
    opt.load_state_dict(saved)
    opt.step()
    assert torch.equal(half, p.detach().half())
    twin_p, twin = copying.deepcopy((p, opt))
    twin_p = twin.param_groups[0]["params"][0]
    twin_p.grad = p.grad.clone()
    opt.step()
    twin.step()
    assert torch.equal(twin_p, p) and torch.equal(twin.param_groups[0]["copies"][0], half)


def test_adamw_on_another_stream():
    """A plan that one stream made serves steps on another, and its memory is not given away while they run."""
    torch.manual_seed(6)
    start = torch.randn(1 << 20, device="cuda")
    grad = torch.randn(1 << 20, device="cuda")
    ends = []
    for streams in ((None, None, None), (None, torch.cuda.Stream(), torch.cuda.Stream())):
        p = torch.nn.Parameter(start.clone())
        opt = AdamW([p], lr=1e-2)
        p.grad = grad.clone()
        before = torch.cuda.current_stream()
        for stream in streams:
            stream = stream or torch.cuda.current_stream()
            stream.wait_stream(before)
            with torch.cuda.stream(stream):
                opt.step()
            before = stream
        opt._plans.clear()
        torch.cuda.current_stream().wait_stream(before)
        ends.append(p.detach().clone())
    assert torch.equal(ends[0], ends[1])


def test_adamw_refuses():
    p = torch.nn.Parameter(torch.zeros(4, device="cuda"))
    with pytest.raises(RuntimeError):
        AdamW([torch.nn.Parameter(torch.zeros(4))])
    with pytest.raises(TypeError):
        AdamW([torch.nn.Parameter(torch.zeros(4, device="cuda", dtype=torch.float64))])
    with pytest.raises(ValueError):
        AdamW([p], states="float4")
    with pytest.raises(ValueError):
        AdamW([{"params": [p], "copies": []}])
    opt = AdamW([p])
    opt.step()                                   # nothing to do
    p.grad = torch.zeros(8, device="cuda")[::2]
    with pytest.raises(TypeError):
        opt.step()


@pytest.mark.parametrize("states", ["float32", "float8"])
def test_the_example_trains_and_serves(states):
    path = os.path.join(H.__file__, "..", "..", "examples", "qat_linear.py")
    spec = importlib.util.spec_from_file_location("qat_linear", os.path.abspath(path))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    losses, off = module.main(steps=150, states=states, tokens=512)
    assert losses[-10:].mean() < 0.3 * losses[0]
    # With the learned scales the second layer's input codes differ from training's only where rounding of the first layer's
    # output (2^-22) crosses a half: fewer than one code in a thousand, a step of 4/127 each.  By token every input has its
    # own rounding, a step of largest/127: about 4 / 127 / sqrt(12) = 0.9 % of the inputs' norm, twice.
    assert off["learned scales"] < 1e-3 and off["scales by token"] < 5e-2

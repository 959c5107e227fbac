"""Offsets beyond 32 bits: rows of the int8 linear layer far apart, a tensor of more than 2^31 elements in the AdamW step."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,k", [(3, 512), (3, 500), (20, 512)])
def test_rows_gigabytes_apart(m, k):
    H.say("linear, rows of %d x %d gigabytes apart" % (m, k))
    rng = np.random.Generator(np.random.Philox(k))
    n = 40
    x, w = rng.standard_normal((m, k)).astype(np.float16), rng.integers(-127, 128, (n, k)).astype(np.int8)
    ws, b = rng.uniform(1e-3, 2e-3, n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    far = 1500000000 if m == 3 else 250000016               # elements; the last row begins behind 2^31 of them
    xd = torch.as_strided(torch.empty((m - 1) * far + k, dtype=torch.float16, device="cuda"), (m, k), (far, 1))
    yd = torch.as_strided(torch.empty((m - 1) * far + n, dtype=torch.float16, device="cuda"), (m, n), (far, 1))
    wd = torch.as_strided(torch.empty((n - 1) * 60000016 + k, dtype=torch.int8, device="cuda"), (n, k), (60000016, 1))
    xd.copy_(H.dev(x))
    wd.copy_(H.dev(w))
    d = fq.FqLinear.from_torch(xd, wd, H.dev(ws), yd, bias=H.dev(b))
    work = torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    fq.fq_linear_forward(d, work)
    torch.cuda.synchronize()
    q, s = R.quantize_rows(x)
    y, off = R.linear(q, s, w, ws, b, True)
    R.check_linear(yd.cpu().numpy(), y, off, True, "far")


@pytest.mark.parametrize("k,n,codes", [(8, 3, False), (16, 16, False), (9, 5, True)])
def test_more_rows_than_a_launch_takes(k, n, codes):
    m = (1 << 23) + 21
    H.say("linear, %d rows of %d" % (m, k))
    gen = torch.Generator(device="cuda").manual_seed(k)
    x = torch.randn((m, k), generator=gen, device="cuda").to(torch.float16)
    q, s = x, None
    if codes:
        q = torch.randint(-127, 128, (m, k), generator=gen, device="cuda", dtype=torch.int8)
        s = torch.rand(m, generator=gen, device="cuda") + 0.5
    rng = np.random.Generator(np.random.Philox(n))
    w = rng.integers(-127, 128, (n, k)).astype(np.int8)
    ws, b = rng.uniform(1e-3, 2e-3, n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    y = torch.full((m, n), 7.0, device="cuda")
    d = fq.FqLinear.from_torch(q, H.dev(w), H.dev(ws), y, bias=H.dev(b), x_scale=s)
    fq.fq_linear_forward(d, torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for part in (slice(0, 300), slice((1 << 23) - 150, m)):
        xq, xs = (q[part].cpu().numpy(), s[part].cpu().numpy()) if codes else R.quantize_rows(x[part].cpu().numpy())
        want, off = R.linear(xq, xs, w, ws, b, False)
        R.check_linear(y[part].cpu().numpy(), want, off, False, "rows %d to %d" % (part.start, part.stop))


def test_a_tensor_of_more_than_two_billion_elements():
    n = (1 << 31) + 777
    H.say("adamw, %d elements" % n)
    zeros = lambda dtype: torch.zeros(n, dtype=dtype, device="cuda")     # noqa: E731
    p, g = zeros(torch.float16), zeros(torch.float16)
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = (torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))
    first = torch.zeros(3, device="cuda")                                # (a list of two: the places are not the indexes)
    rng = np.random.Generator(np.random.Philox(1))
    parts = [slice(0, 1000), slice((1 << 31) - 512, (1 << 31) + 300), slice((n - 1000) // 256 * 256, n)]
    for part in parts[:2] + [slice(parts[2].start + 256, n)]:
        count = part.stop - part.start
        p[part] = H.dev(rng.standard_normal(count).astype(np.float16))
        g[part] = H.dev(rng.standard_normal(count).astype(np.float16))
    params = [fq.FqParam.from_torch(first, first.clone(), torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda")),
              fq.FqParam.from_torch(p, g, m, v, ms, vs, weight_decay=0.1)]
    work = torch.empty(fq.fq_adamw_workspace_bytes(params), dtype=torch.uint8, device="cuda")
    plan = fq.fq_adamw_create(params, work)
    h = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, step=3, seed=5)
    before = [(p[s].cpu().numpy(), g[s].cpu().numpy()) for s in parts]
    fq.fq_adamw_step(plan, fq.FqAdamW(**h))
    torch.cuda.synchronize()
    for s, (p0, g0) in zip(parts, before):
        count = s.stop - s.start
        blocks = slice(s.start // 256, (s.stop + 255) // 256)
        zero, none = np.zeros(count, np.float32), np.zeros(blocks.stop - blocks.start, np.float32)
        want = R.step(p0, g0, zero, zero, none, none, h, 256 + s.start, 1.0, 0.1)
        whole = count if s.stop == n else count // 256 * 256              # (a last block that goes on has another scale)
        got = p[s].cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - want["p"]) <= want["off"])
        assert np.array_equal(m[s].float().cpu().numpy()[:whole], want["m8"].astype(np.float32)[:whole])
        code = v[s].float().cpu().numpy().astype(np.float64)[:whole]
        assert np.all((code >= want["v8_least"][:whole]) & (code <= want["v8_most"][:whole]))
    assert float(p[2000:3000].abs().max()) == 0.0 and float(m[1 << 30:(1 << 30) + 4096].float().abs().max()) == 0.0
    fq.fq_adamw_destroy(plan)

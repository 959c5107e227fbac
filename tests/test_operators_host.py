"""What fq_linear and fq_adamw refuse and how they size their workspaces: host logic, no GPU call."""
import ctypes

import numpy as np
import pytest

from paper_2511_12653_amd import binding as fq

import _operators_ref as R

A = 1 << 20                      # addresses that nothing touches


def linear(**kw):
    base = dict(m=40, n=30, k=100, x_dtype=fq.FQ_F16, y_dtype=fq.FQ_F16, ldx=100, ldw=100, ldy=30, x=A, xs=None, w=2 * A, ws=3 * A,
                bias=None, y=4 * A, xs_step=1, ws_step=1)
    base.update(kw)
    return fq.FqLinear(**base)


def status(d, workspace=5 * A, nbytes=1 << 30):
    return fq._lib.fq_linear_forward(ctypes.byref(d), workspace, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x_dtype=3), -2), (dict(y_dtype=2), -2), (dict(x_dtype=-1), -2),
    (dict(m=-1), -3), (dict(n=-1), -3), (dict(k=-1), -3), (dict(k=131072, ldx=131072, ldw=131072), -3), (dict(m=1 << 31), -3),
    (dict(ldx=99), -3), (dict(ldw=99), -3), (dict(ldy=29), -3), (dict(ldx=1 << 60), -3), (dict(ws_step=2), -3), (dict(xs_step=-1), -3),
    (dict(x=None), -1), (dict(w=None), -1), (dict(ws=None), -1), (dict(y=None), -1), (dict(x_dtype=2, xs=None), -1),
    (dict(x=A + 1), -5), (dict(ws=3 * A + 2), -5), (dict(bias=3 * A + 1), -5), (dict(y=4 * A + 1), -5),
    (dict(x_dtype=1, x=A + 2), -5), (dict(y_dtype=1, y=4 * A + 2), -5), (dict(x_dtype=2, xs=A + 1), -5),
    (dict(y=A), -9), (dict(y=A + 2 * 100 * 39 + 2 * 99), -9), (dict(y=2 * A - 2), -9), (dict(y=3 * A + 116), -9),
    (dict(bias=4 * A + 2396), -9), (dict(x_dtype=2, xs=4 * A), -9)])
def test_linear_refuses(kw, code):
    d = linear(**kw)
    assert status(d) == code
    assert fq.fq_linear_workspace_bytes(d) == 0
    with pytest.raises(fq.FqError) as e:
        fq.fq_linear_forward(d, (5 * A, 1 << 30), stream=ctypes.c_void_p())
    assert e.value.status == code


def test_linear_workspace():
    assert fq._lib.fq_linear_forward(None, None, 0, None) == -1 and fq._lib.fq_linear_workspace_bytes(None) == 0
    d = linear()
    nbytes = fq.fq_linear_workspace_bytes(d)
    assert nbytes >= 40 * 100 + 40 * 4 and nbytes % 256 == 0
    assert status(d, None, 0) == -6 and status(d, 5 * A, nbytes - 1) == -6 and status(d, 5 * A + 128, nbytes) == -5
    for kw in (dict(m=0), dict(n=0, ldy=0), dict(m=0, x=None, w=None, ws=None, y=None)):     # nothing to do: no launch, no workspace
        assert status(linear(**kw), None, 0) == 0 and fq.fq_linear_workspace_bytes(linear(**kw)) >= 256


def test_linear_columns_of_one_buffer_do_not_overlap():
    # x: columns 8..107 of rows of 160 FP16 values, y: columns 108..137; then one column less, and y in front of x
    ok = dict(ldx=160, ldy=160, x=A + 16)
    assert fq.fq_linear_workspace_bytes(linear(y=A + 216, **ok)) > 0
    assert fq.fq_linear_workspace_bytes(linear(y=A + 214, **ok)) == 0
    assert fq.fq_linear_workspace_bytes(linear(y=A + 216, **dict(ok, ldy=161))) == 0
    assert fq.fq_linear_workspace_bytes(linear(y=A + 320 + 276, **ok)) > 0 and fq.fq_linear_workspace_bytes(linear(y=A + 320 + 278, **ok)) == 0       # runs into the next row's x
    assert fq.fq_linear_workspace_bytes(linear(ldx=160, ldy=160, y=A, x=A + 60)) > 0
    assert fq.fq_linear_workspace_bytes(linear(ldx=160, ldy=160, y=A, x=A + 58)) == 0


def param(**kw):
    base = dict(n=1000, p_dtype=fq.FQ_F32, g_dtype=fq.FQ_F32, state=fq.FQ_STATE_F8, lr_scale=1.0, weight_decay=0.0, p=A, g=2 * A,
                p16=None, m=3 * A, v=4 * A, m_scale=5 * A, v_scale=6 * A)
    base.update(kw)
    return fq.FqParam(**base)


def create(params, workspace=7 * A, nbytes=1 << 20):
    plan = ctypes.c_void_p(123)
    arr = (fq.FqParam * max(1, len(params)))(*params)
    st = fq._lib.fq_adamw_create(arr, len(params), workspace, nbytes, None, ctypes.byref(plan))
    return st, plan


@pytest.mark.parametrize("kw,code", [
    (dict(p_dtype=2), -2), (dict(g_dtype=7), -2), (dict(state=2), -2), (dict(p_dtype=fq.FQ_F16, p16=8 * A), -2),
    (dict(n=-1), -3), (dict(n=1 << 41), -3), (dict(lr_scale=float("nan")), -10), (dict(weight_decay=float("inf")), -10),
    (dict(p=None), -1), (dict(g=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(m_scale=None), -1), (dict(v_scale=None), -1),
    (dict(p=A + 2), -5), (dict(g=2 * A + 1), -5), (dict(state=0, m=3 * A + 2), -5), (dict(v_scale=6 * A + 1), -5), (dict(p16=8 * A + 1), -5),
    (dict(g=A), -9), (dict(g=A + 3996), -9), (dict(m=4 * A), -9), (dict(v_scale=5 * A + 12), -9), (dict(p16=A + 2000), -9),
    (dict(m_scale=3 * A + 996), -9)])
def test_adamw_refuses(kw, code):
    st, plan = create([param(n=0), param(**kw)])
    assert st == code and plan.value is None
    assert fq.fq_adamw_workspace_bytes([param(), param(**kw)]) == 0


def test_adamw_workspace_and_empty_lists():
    nbytes = fq.fq_adamw_workspace_bytes([param()] * 5)
    assert nbytes % 256 == 0 and nbytes > 0
    assert create([param()] * 5, None)[0] == -6 and create([param()] * 5, 7 * A, nbytes - 1)[0] == -6
    assert create([param()] * 5, 7 * A + 8)[0] == -5
    assert fq._lib.fq_adamw_create(None, 3, None, 0, None, ctypes.byref(ctypes.c_void_p())) == -1
    assert fq._lib.fq_adamw_create(None, -1, None, 0, None, ctypes.byref(ctypes.c_void_p())) == -3
    assert fq._lib.fq_adamw_create(None, 0, None, 0, None, None) == -1
    for params in ([], [param(n=0, p=None, g=None, m=None, v=None, m_scale=None, v_scale=None)] * 3):
        st, plan = create(params, None, 0)
        assert st == 0 and plan.value
        h = fq.FqAdamW()
        assert fq._lib.fq_adamw_step(plan, ctypes.byref(h), None) == 0           # no launch
        for kw in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(beta2=float("nan")), dict(lr=float("inf")), dict(eps=-1e-8),
                   dict(eps=float("nan"))):
            h = fq.FqAdamW(**kw)
            assert fq._lib.fq_adamw_step(plan, ctypes.byref(h), None) == -10
        h = fq.FqAdamW()
        h.grad_scale = A + 2
        assert fq._lib.fq_adamw_step(plan, ctypes.byref(h), None) == -5
        assert fq._lib.fq_adamw_step(plan, None, None) == -1 and fq._lib.fq_adamw_step(None, ctypes.byref(h), None) == -1
        fq.fq_adamw_destroy(plan)
    fq.fq_adamw_destroy(None)


def test_structures_match_the_header():
    assert ctypes.sizeof(fq.FqLinear) == 3 * 8 + 8 + 3 * 8 + 6 * 8 + 8
    assert ctypes.sizeof(fq.FqParam) == 8 + 3 * 4 + 2 * 4 + 4 + 7 * 8
    assert ctypes.sizeof(fq.FqAdamW) == 4 * 8 + 3 * 8


def test_tensors_on_the_host_are_refused():
    import torch
    t = torch.zeros(4)
    with pytest.raises(ValueError):
        fq.FqParam.from_torch(t, t, t, t)
    with pytest.raises(TypeError):
        fq.FqParam.from_torch(t.double(), t, t, t)
    with pytest.raises(ValueError):
        fq.FqLinear.from_torch(torch.zeros(2, 3), torch.zeros(4, 3, dtype=torch.int8), torch.zeros(4), torch.zeros(2, 4))
    with pytest.raises(ValueError):
        fq.FqAdamW(grad_scale=torch.ones(1))


def test_the_random_bits_are_uniform_and_independent():
    """Mean, spread and correlation of the 16-bit halves: between the halves, neighbours, blocks and steps, to five
    standard deviations; all 32 bits are one half of the time set."""
    n = 1 << 20
    at = np.arange(n, dtype=np.uint64)
    x, y = R.random_bits(at, R.key(3, 1)), R.random_bits(at, R.key(3, 2))
    series = [x & np.uint64(0xFFFF), x >> np.uint64(16), y & np.uint64(0xFFFF), y >> np.uint64(16)]
    unit = [(s.astype(np.float64) + 0.5) / 65536 - 0.5 for s in series]
    for u in unit:
        assert abs(u.mean()) <= 5 * np.sqrt(1 / 12 / n) and abs(u.var() * 12 - 1) <= 5 * np.sqrt(0.8 / n)
        for lag in (1, 2, 4, 64, 256, 1024):
            assert abs((u[lag:] * u[:-lag]).mean() * 12) <= 5 / np.sqrt(n - lag)
    for i in range(4):
        for j in range(i):
            assert abs((unit[i] * unit[j]).mean() * 12) <= 5 / np.sqrt(n)
    for bit in range(32):
        assert abs(((x >> np.uint64(bit)) & np.uint64(1)).astype(np.float64).mean() - 0.5) <= 5 * 0.5 / np.sqrt(n)

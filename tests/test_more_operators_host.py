"""What fq_norm, fq_dropout and fq_adapters refuse and how they size their workspaces: host logic, no GPU call."""
import ctypes
import math

import numpy as np
import pytest

from paper_2511_12653_amd import binding as fq

import _more_operators_ref as R

A = 1 << 24                      # addresses that nothing touches


def norm(**kw):
    base = dict(rows=40, width=100, x_dtype=fq.FQ_F16, y_dtype=fq.FQ_F16, w_dtype=fq.FQ_F32, eps=1e-5, ldx=100, ldy=100, ldgy=100,
                ldgx=100, x=A, weight=2 * A, bias=3 * A, y=4 * A, ys=None, stats=5 * A, gy=6 * A, gx=7 * A, gweight=8 * A, gbias=9 * A)
    base.update(kw)
    return fq.FqNorm(**base)


def forward(d):
    return fq._lib.fq_norm_forward(ctypes.byref(d), None)


def backward(d, workspace=10 * A, nbytes=1 << 30):
    return fq._lib.fq_norm_backward(ctypes.byref(d), workspace, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x_dtype=2), -2), (dict(x_dtype=-1), -2), (dict(y_dtype=3), -2), (dict(w_dtype=2), -2),
    (dict(rows=-1), -3), (dict(width=-1), -3), (dict(width=(1 << 24) + 1, ldx=1 << 25, ldy=1 << 25), -3), (dict(rows=(1 << 36) + 1), -3),
    (dict(ldx=99), -3), (dict(ldy=99), -3), (dict(ldx=1 << 60), -3),
    (dict(eps=-1e-9), -7), (dict(eps=math.nan), -7), (dict(eps=math.inf), -7),
    (dict(x=A + 1), -5), (dict(weight=2 * A + 2), -5), (dict(bias=3 * A + 2), -5), (dict(y=4 * A + 1), -5), (dict(stats=5 * A + 2), -5),
    (dict(x_dtype=1, x=A + 2), -5), (dict(y_dtype=2, ys=8 * A + 1), -5), (dict(w_dtype=0, bias=3 * A + 1), -5),
    (dict(x=None), -1), (dict(y=None), -1), (dict(y_dtype=2, ys=None), -1),
    (dict(y=A + 2), -9), (dict(y=A, ldy=101), -9), (dict(y=A, y_dtype=1), -9), (dict(y=A + 2 * 3999), -9), (dict(y=2 * A), -9), (dict(y=3 * A + 396), -9),
    (dict(stats=4 * A), -9), (dict(stats=A + 4), -9), (dict(stats=2 * A), -9), (dict(y_dtype=2, ys=4 * A), -9), (dict(y_dtype=2, ys=5 * A), -9),
    (dict(y_dtype=2, ys=A), -9)])
def test_norm_forward_refuses(kw, code):
    assert forward(norm(**kw)) == code
    with pytest.raises(fq.FqError) as e:
        fq.fq_norm_forward(norm(**kw), stream=ctypes.c_void_p())
    assert e.value.status == code


@pytest.mark.parametrize("kw,code", [
    (dict(y_dtype=2), -2), (dict(x_dtype=2), -2), (dict(w_dtype=5), -2), (dict(rows=-1), -3), (dict(ldgy=99), -3), (dict(ldgx=99), -3), (dict(ldx=0), -3),
    (dict(eps=-1.0), -7), (dict(gy=6 * A + 1), -5), (dict(gx=7 * A + 1), -5), (dict(gweight=8 * A + 2), -5), (dict(gbias=9 * A + 1), -5), (dict(stats=5 * A + 1), -5),
    (dict(x=None), -1), (dict(gy=None), -1), (dict(stats=None), -1),
    (dict(gx=A + 2), -9), (dict(gx=6 * A, ldgx=120), -9), (dict(gx=2 * A), -9), (dict(gx=5 * A), -9), (dict(gweight=A), -9), (dict(gweight=9 * A), -9),
    (dict(gbias=7 * A + 8), -9), (dict(gweight=2 * A), -9), (dict(gbias=5 * A + 4), -9), (dict(gweight=6 * A), -9)])
def test_norm_backward_refuses(kw, code):
    d = norm(**kw)
    assert backward(d) == code and fq.fq_norm_workspace_bytes(d) == 0
    with pytest.raises(fq.FqError) as e:
        fq.fq_norm_backward(d, (10 * A, 1 << 30), stream=ctypes.c_void_p())
    assert e.value.status == code


def test_norm_workspace_and_nothing_to_do():
    assert fq._lib.fq_norm_forward(None, None) == -1 and fq._lib.fq_norm_backward(None, None, 0, None) == -1
    assert fq._lib.fq_norm_workspace_bytes(None) == 0
    nbytes = fq.fq_norm_workspace_bytes(norm())
    assert nbytes % 256 == 0 and nbytes >= 2 * 100 * 4
    assert backward(norm(), None, 0) == -6 and backward(norm(), 10 * A, nbytes - 1) == -6 and backward(norm(), 10 * A + 64, nbytes) == -5
    for kw in (dict(rows=0), dict(width=0), dict(rows=0, x=None, y=None, stats=None)):
        assert forward(norm(**kw)) == 0
    for kw in (dict(width=0), dict(rows=0, gweight=None, gbias=None), dict(gx=None, gweight=None, gbias=None)):
        assert backward(norm(**kw), None, 0) == 0
    for kw in (dict(gx=A), dict(gx=6 * A), dict(gx=None), dict(weight=None), dict(gweight=None), dict(y=None, ldy=0)):
        assert fq.fq_norm_workspace_bytes(norm(**kw)) > 0
    # no more than 1 % of the traffic goes to partial sums where rows are many, and the parts of wide rows stay few
    assert fq.fq_norm_workspace_bytes(norm(rows=1 << 20, width=4096, ldx=4096, ldgy=4096, ldgx=4096)) < 1 << 30
    wide = dict(rows=4096, width=1 << 24, ldx=1 << 24, ldgy=1 << 24, ldgx=1 << 24, gx=None, x=1 << 44, gy=1 << 45, weight=None)
    assert 0 < fq.fq_norm_workspace_bytes(norm(**dict(wide, gweight=1 << 50, gbias=1 << 51))) <= 16 * 2 * 4 << 24


def dropout(**kw):
    base = dict(n=1000, x_dtype=fq.FQ_F16, y_dtype=fq.FQ_F16, p=0.1, seed=1, step=2, step_on_device=None, x=A, residual=2 * A, y=3 * A)
    base.update(kw)
    return fq.FqDropout(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(x_dtype=2), -2), (dict(y_dtype=-1), -2), (dict(n=-1), -3), (dict(n=(1 << 35) + 1), -3),
    (dict(p=-1e-9), -7), (dict(p=1.0000001), -7), (dict(p=math.nan), -7),
    (dict(x=A + 1), -5), (dict(residual=2 * A + 1), -5), (dict(y=3 * A + 1), -5), (dict(step_on_device=4 * A + 4), -5), (dict(y_dtype=1, y=3 * A + 2), -5),
    (dict(x=None), -1), (dict(y=None), -1),
    (dict(y=A + 2), -9), (dict(y=A - 2), -9), (dict(y=2 * A + 1998), -9), (dict(y=A, y_dtype=1), -9), (dict(step_on_device=3 * A + 1992), -9)])
def test_dropout_refuses(kw, code):
    assert fq._lib.fq_dropout(ctypes.byref(dropout(**kw)), None) == code
    with pytest.raises(fq.FqError) as e:
        fq.fq_dropout(dropout(**kw), stream=ctypes.c_void_p())
    assert e.value.status == code


def test_dropout_of_nothing():
    assert fq._lib.fq_dropout(None, None) == -1
    assert fq._lib.fq_dropout(ctypes.byref(dropout(n=0, x=None, y=None, residual=None)), None) == 0


def adapters(**kw):
    base = dict(m=40, n=30, k=100, count=3, rank=8, x_dtype=fq.FQ_F16, y_dtype=fq.FQ_F16, base_dtype=fq.FQ_F16, xs_step=1, ldx=100, ldy=30,
                ldbase=30, x=A, xs=None, ids=2 * A, a=3 * A, b=4 * A, scale=5 * A, base=6 * A, y=7 * A)
    base.update(kw)
    return fq.FqAdapters(**base)


def apply(d, workspace=8 * A, nbytes=1 << 30):
    return fq._lib.fq_adapters_forward(ctypes.byref(d), workspace, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x_dtype=3), -2), (dict(y_dtype=2), -2), (dict(base_dtype=2), -2),
    (dict(m=-1), -3), (dict(n=-1), -3), (dict(k=-1), -3), (dict(count=-1), -3), (dict(rank=-1), -3), (dict(rank=257), -3), (dict(m=1 << 31), -3),
    (dict(k=(1 << 20) + 1, ldx=1 << 21), -3), (dict(n=(1 << 20) + 1, ldy=1 << 21, ldbase=1 << 21), -3), (dict(count=1 << 31), -3),
    (dict(ldx=99), -3), (dict(ldy=29), -3), (dict(ldbase=29), -3), (dict(xs_step=2), -3), (dict(ldy=1 << 60), -3),
    (dict(x=A + 1), -5), (dict(ids=2 * A + 2), -5), (dict(a=3 * A + 1), -5), (dict(b=4 * A + 1), -5), (dict(scale=5 * A + 2), -5), (dict(base=6 * A + 1), -5),
    (dict(y=7 * A + 1), -5), (dict(x_dtype=2, xs=8 * A + 2), -5), (dict(x_dtype=1, x=A + 2), -5), (dict(base_dtype=1, base=6 * A + 2), -5),
    (dict(x=None), -1), (dict(ids=None), -1), (dict(a=None), -1), (dict(b=None), -1), (dict(y=None), -1), (dict(x_dtype=2), -1),
    (dict(y=6 * A + 2), -9), (dict(y=6 * A, ldy=40), -9), (dict(y=6 * A, base_dtype=1), -9), (dict(y=A), -9), (dict(y=2 * A), -9), (dict(y=3 * A + 100), -9),
    (dict(y=4 * A + 2 * 30 * 8 * 3 - 2), -9), (dict(y=5 * A + 8), -9), (dict(x_dtype=2, xs=7 * A + 4), -9)])
def test_adapters_refuse(kw, code):
    d = adapters(**kw)
    assert apply(d) == code and fq.fq_adapters_workspace_bytes(d) == 0
    with pytest.raises(fq.FqError) as e:
        fq.fq_adapters_forward(d, (8 * A, 1 << 30), stream=ctypes.c_void_p())
    assert e.value.status == code


def test_adapters_workspace_and_nothing_to_do():
    assert fq._lib.fq_adapters_forward(None, None, 0, None) == -1 and fq._lib.fq_adapters_workspace_bytes(None) == 0
    nbytes = fq.fq_adapters_workspace_bytes(adapters())
    assert nbytes % 256 == 0 and nbytes >= 40 * 8 * 4
    assert apply(adapters(), None, 0) == -6 and apply(adapters(), 8 * A, nbytes - 1) == -6 and apply(adapters(), 8 * A + 128, nbytes) == -5
    for kw in (dict(m=0), dict(n=0, ldy=0, ldbase=0), dict(m=0, x=None, y=None, a=None, b=None, ids=None)):
        assert apply(adapters(**kw), None, 0) == 0
    for kw in (dict(y=6 * A), dict(base=None), dict(scale=None), dict(count=0, a=None, b=None), dict(rank=0, a=None, b=None), dict(k=0, x=None, a=None, ldx=0)):
        assert fq.fq_adapters_workspace_bytes(adapters(**kw)) > 0


def test_structures_match_the_header():
    assert ctypes.sizeof(fq.FqNorm) == 2 * 8 + 4 * 4 + 4 * 8 + 10 * 8
    assert ctypes.sizeof(fq.FqDropout) == 8 + 2 * 4 + 8 + 2 * 8 + 4 * 8
    assert ctypes.sizeof(fq.FqAdapters) == 5 * 8 + 4 * 4 + 3 * 8 + 8 * 8


def test_from_torch_refuses():
    import torch
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t)     # noqa: E731
    x = z(4, 6)
    for bad in (lambda: fq.FqNorm.from_torch(x), lambda: fq.FqNorm.from_torch(x, y=x), lambda: fq.FqNorm.from_torch(x, y=z(4, 5)),
                lambda: fq.FqNorm.from_torch(x, y=z(4, 6, t=torch.int8)), lambda: fq.FqNorm.from_torch(x, y=x, y_scale=z(4, t=torch.float32)),
                lambda: fq.FqNorm.from_torch(x, y=x, weight=z(5)), lambda: fq.FqNorm.from_torch(x, y=x, stats=z(4, 1, t=torch.float32)),
                lambda: fq.FqNorm.from_torch(z(4, 3, 2), y=z(4, 3, 2)), lambda: fq.FqDropout.from_torch(x, z(5, 6), 0.1, 1),
                lambda: fq.FqDropout.from_torch(x, x, 0.1, -1), lambda: fq.FqDropout.from_torch(x, x, 0.1, 1, 1 << 64),
                lambda: fq.FqDropout.from_torch(x, x, 0.1, 1),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int32), z(2, 3, 6), z(2, 8, 3), z(4, 8)),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int32), z(2, 3, 5), z(2, 8, 3), z(4, 8)),
                lambda: fq.FqAdapters.from_torch(x, z(3, t=torch.int32), z(2, 3, 6), z(2, 8, 3), z(4, 8)),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int32), z(2, 3, 6), z(2, 8, 4), z(4, 8)),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int32), z(2, 3, 6), z(2, 8, 3), z(4, 8), scale=z(1, t=torch.float32)),
                lambda: fq.FqAdapters.from_torch(x.to(torch.int8), z(4, t=torch.int32), z(2, 3, 6), z(2, 8, 3), z(4, 8))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: fq.FqNorm.from_torch(x.double(), y=x), lambda: fq.FqNorm.from_torch(x, y=x.double()),
                lambda: fq.FqNorm.from_torch(x, gy=x.to(torch.int8)), lambda: fq.FqNorm.from_torch(x, y=x, gy=x.float()),
                lambda: fq.FqNorm.from_torch(x, y=x, weight=z(6), bias=z(6, t=torch.float32)), lambda: fq.FqNorm.from_torch(x, gy=x, gx=x.float()),
                lambda: fq.FqNorm.from_torch(x, y=x, stats=z(4, 2)), lambda: fq.FqDropout.from_torch(x.double(), x, 0.1, 1),
                lambda: fq.FqDropout.from_torch(x, x, 0.1, 1, residual=x.float()), lambda: fq.FqDropout.from_torch(x, x, 0.1, 1, step_on_device=z(1)),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int64), z(2, 3, 6), z(2, 8, 3), z(4, 8)),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int32), z(2, 3, 6, t=torch.float32), z(2, 8, 3), z(4, 8)),
                lambda: fq.FqAdapters.from_torch(x, z(4, t=torch.int32), z(2, 3, 6), z(2, 8, 3), z(4, 8), scale=z(2))):
        with pytest.raises(TypeError):
            bad()


def test_the_masks_are_uniform_and_independent():
    """The 31 bits: mean, spread and correlation with neighbours, at strides, between steps and between seeds, to five standard
    deviations; every bit is set one half of the time; and masks of two steps are no shifted copies of each other."""
    n = 1 << 20
    at = np.arange(n, dtype=np.uint64)
    series = [R.random_bits(at, seed, step).astype(np.float64) / 2.0 ** 31 - 0.5 for seed, step in ((3, 0), (3, 1), (4, 0), (3, 1 << 33))]
    series.append(R.random_bits(at + np.uint64(1 << 32), 3, 0).astype(np.float64) / 2.0 ** 31 - 0.5)
    for u in series:
        assert abs(u.mean()) <= 5 * np.sqrt(1 / 12 / n) and abs(u.var() * 12 - 1) <= 5 * np.sqrt(0.8 / n)
        for lag in (1, 2, 3, 4, 8, 64, 256, 384, 1024, 4096, 65536):
            assert abs((u[lag:] * u[:-lag]).mean() * 12) <= 5 / np.sqrt(n - lag), lag
    for i in range(len(series)):
        for j in range(i):
            assert abs((series[i] * series[j]).mean() * 12) <= 5 / np.sqrt(n)
    x = R.random_bits(at, 3, 0)
    for bit in range(31):
        assert abs(((x >> np.uint64(bit)) & np.uint64(1)).astype(np.float64).mean() - 0.5) <= 5 * 0.5 / np.sqrt(n)
    # values of one step that occur in another's: 2^20 of 2^31 values, so 2^20 * 2^20 / 2^31 pairs = 512 are expected; of those that do
    # occur, no two at one distance where the second key moves them
    y = R.random_bits(at, 3, 1)
    common, ix, iy = np.intersect1d(x, y, return_indices=True)
    distance = ix.astype(np.int64) - iy
    assert common.size < 2000 and np.unique(distance, return_counts=True)[1].max() <= 3
    for p in (0.1, 0.5, 0.9):
        kept = R.keep(n, p, 8, 8).mean()
        assert abs(kept - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / n)

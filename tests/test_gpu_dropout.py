"""fq_dropout against the plain implementation, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _more_operators_ref as R

pytestmark = pytest.mark.gpu


def values(n, dtype, seed):
    return np.random.Generator(np.random.Philox(seed)).standard_normal(n).astype(dtype)


def run(x, p, seed, step, residual, y_type, shift=0, on_device=None):
    place = lambda a: torch.cat([torch.zeros(shift, device="cuda", dtype=H.dev(a[:0]).dtype), H.dev(a)])[shift:]     # noqa: E731
    buf = torch.full((x.size + 16 + shift,), 77, device="cuda", dtype=torch.float16 if y_type == np.float16 else torch.float32)
    y = buf[shift:shift + x.size]
    d = fq.FqDropout.from_torch(place(x), y, p, seed, step, None if residual is None else place(residual),
                                None if on_device is None else torch.tensor([on_device], device="cuda"))
    fq.fq_dropout(d)
    torch.cuda.synchronize()
    assert (buf[shift + x.size:] == 77).all() and (buf[:shift] == 77).all()
    return y.cpu().numpy()


@pytest.mark.parametrize("x_type,y_type", [(np.float16, np.float16), (np.float16, np.float32), (np.float32, np.float16), (np.float32, np.float32)])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 100, 2047, 2048, 2049, 4095, 4096, 4104, 100003])
def test_values(n, x_type, y_type):
    x, r = values(n, x_type, n), values(n, y_type, n + 1)
    for p in (0.0, 0.1, 0.5, 0.999, 1.0):
        for residual in (None, r):
            for shift in (0, 1):
                got = run(x, p, 5 + n, 3, residual, y_type, shift)
                want = R.dropout(x, p, 5 + n, 3, residual, y_type == np.float16)
                assert np.array_equal(got.view(np.uint8), want.view(np.uint8)), (p, residual is None, shift)


@pytest.mark.parametrize("seed,step", [(0, 0), ((1 << 64) - 1, 0), (1 << 63, (1 << 64) - 1), (12345678901234567890, 1 << 40)])
def test_seeds_and_steps(seed, step):
    x = values(5000, np.float32, 1)
    assert np.array_equal(run(x, 0.3, seed, step, None, np.float32), R.dropout(x, 0.3, seed, step, None, False))
    # the step on the GPU is added, modulo 2^64
    assert np.array_equal(run(x, 0.3, seed, step, None, np.float32, on_device=7),
                          R.dropout(x, 0.3, seed, (step + 7) % (1 << 64), None, False))


def test_what_is_dropped_does_not_count():
    x = values(4096, np.float32, 2)
    kept = R.keep(x.size, 0.5, 9, 0)
    x[~kept] = np.nan
    x[np.nonzero(~kept)[0][::3]] = np.inf
    got = run(x, 0.5, 9, 0, None, np.float32)
    assert np.isfinite(got).all() and (got[~kept] == 0).all()
    assert (run(x, 1.0, 9, 0, None, np.float32) == 0).all()


def test_in_place():
    x, r = values(10001, np.float16, 3), values(10001, np.float16, 4)
    want = R.dropout(x, 0.2, 1, 2, r, True)
    for which in (0, 1):
        xd, rd = H.dev(x), H.dev(r)
        fq.fq_dropout(fq.FqDropout.from_torch(xd, (xd, rd)[which], 0.2, 1, 2, rd))
        assert np.array_equal((xd, rd)[which].cpu().numpy(), want)


def test_places_beyond_32_bits():
    """The 2^32nd element begins another sequence: 8.6 GB of FP16, in place, of which a few runs are looked at."""
    n = (1 << 32) + 5001
    x = torch.ones(n, device="cuda", dtype=torch.float16)
    fq.fq_dropout(fq.FqDropout.from_torch(x, x, 0.5, 11, 4))
    for begin, count in ((0, 3000), ((1 << 31) - 100, 200), ((1 << 32) - 4096, 4096), (1 << 32, 5001)):
        assert np.array_equal(x[begin:begin + count].cpu().numpy() != 0, R.keep(count, 0.5, 11, 4, begin)), begin


def test_captured_steps_go_on():
    """A captured call with the step on the GPU makes another mask in every replay: that of the same step made eagerly."""
    x = H.dev(values(20001, np.float32, 6))
    y, step = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda")
    d = fq.FqDropout.from_torch(x, y, 0.25, 77, 100, step_on_device=step)
    fq.fq_dropout(d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.add_(1)
        fq.fq_dropout(d)
    for replay in range(1, 5):
        y.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert int(step) == replay
        assert np.array_equal(y.cpu().numpy(), R.dropout(x.cpu().numpy(), 0.25, 77, 100 + replay, None, False))

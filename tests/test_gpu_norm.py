"""fq_norm_forward and fq_norm_backward against the plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _more_operators_ref as R

pytestmark = pytest.mark.gpu
EPS = 1e-5
WIDTHS = [1, 2, 7, 8, 9, 16, 63, 120, 128, 129, 250, 256, 264, 383, 384, 391, 512, 513, 1000, 1024, 1025, 2047, 2048, 2056, 3001, 4096,
          4104, 5003, 8192, 8200, 12001, 16384]
WIDE = [16385, 16392, 20001, 40000, 65536]


def rng_of(*seed):
    return np.random.Generator(np.random.Philox(list(seed)[0] * 1000003 + sum((i + 1) * 7919 * s for i, s in enumerate(seed[1:]))))


def tokens(rng, rows, width, dtype, mean=0.3):
    x = rng.standard_normal((rows, width)) * np.exp(0.5 * rng.standard_normal((rows, 1))) + mean * rng.standard_normal((rows, 1))
    return x.astype(dtype)


def placed(a, pitch, shift):
    """The matrix on the GPU, in rows `pitch` apart from element `shift` of a buffer on, and the buffer; what is between holds 99."""
    rows, width = a.shape
    flat = torch.full((shift + max(1, rows) * pitch,), 99, dtype=H.dev(a[:0]).dtype, device="cuda")
    view = flat[shift:shift + rows * pitch].view(rows, pitch)[:, :width]
    view.copy_(H.dev(a))
    return view, flat


def forward(x, w, b, y_type, eps=EPS, pitch=0, shift=0, stats=True, in_place=False):
    rows, width = x.shape
    xd, xbuf = placed(x, width + pitch, shift)
    if in_place:
        y, buf = xd, xbuf
    else:
        y, buf = placed(np.full((rows, width), 77, dtype=y_type), width + pitch, shift)
    s = torch.full((rows, 2), 77.0, device="cuda") if stats else None
    ys = torch.full((rows,), 77.0, device="cuda") if y_type == np.int8 else None
    d = fq.FqNorm.from_torch(xd, y=y, weight=None if w is None else H.dev(w), bias=None if b is None else H.dev(b), y_scale=ys, stats=s, eps=eps)
    fq.fq_norm_forward(d)
    torch.cuda.synchronize()
    if pitch:                       # what lies between the rows is as it was
        flat = buf.cpu().numpy()[shift:].reshape(rows, width + pitch)
        assert (flat[:, width:] == 99).all()
    return y.cpu().numpy(), None if s is None else s.cpu().numpy(), None if ys is None else ys.cpu().numpy()


def check_forward(x, w, b, y_type, label, eps=EPS, **kw):
    got, stats, ys = forward(x, w, b, y_type, eps, **kw)
    y, off, mean, rstd = R.norm(x, w, b, eps)
    if stats is not None:
        # binary64 sums of k terms from the row's first value on: k 2^-53 (1 + (x0 - mean)^2 / var) of them, at most 1e-9 here
        fine = np.isfinite(x.astype(np.float64)).all(1)
        R.check(stats[fine, 0], mean[fine], 1e-12 * np.abs(x[fine].astype(np.float64)).max(1, initial=0.0), False, label + " mean")
        R.check(stats[fine, 1], rstd[fine], 1e-9 * rstd[fine], False, label + " rstd")
    if y_type == np.int8:
        q, s, near = R.codes(x, w, b, eps)
        assert np.array_equal(ys, s, equal_nan=True), label + " scales"
        # y in binary64 may differ in its last bits: its binary32 value then by a step, which moves a code where y / s is as near to a half
        sure = near > 127 * 2.0 ** -23
        assert np.array_equal(got[sure], q[sure]) and np.abs(got.astype(int) - q).max(initial=0) <= 1, label + " codes"
        assert (got != q).mean() < 1e-3 if got.size else True
    else:
        R.check(got, y, off, y_type == np.float16, label)


@pytest.mark.parametrize("y_type", [np.float16, np.float32, np.int8])
@pytest.mark.parametrize("x_type", [np.float16, np.float32])
@pytest.mark.parametrize("width", WIDTHS + WIDE)
def test_forward_widths(width, x_type, y_type):
    rng = rng_of(1, width, x_type().itemsize, y_type().itemsize)
    for rows in (1, 5, 67):
        x = tokens(rng, rows, width, x_type)
        w, b = (1 + 0.2 * rng.standard_normal(width)).astype(np.float32), (0.1 * rng.standard_normal(width)).astype(np.float32)
        check_forward(x, w, b, y_type, "%d x %d" % (rows, width))


@pytest.mark.parametrize("w_type", [None, np.float16, np.float32])
@pytest.mark.parametrize("width,pitch,shift", [(40, 0, 1), (40, 1, 0), (384, 8, 8), (384, 3, 5), (1155, 0, 3), (4096, 1, 1), (20000, 7, 1)])
def test_forward_strides_and_weights(width, pitch, shift, w_type):
    rng = rng_of(2, width, pitch, shift)
    for x_type, y_type in ((np.float16, np.float16), (np.float32, np.float16), (np.float16, np.float32), (np.float16, np.int8), (np.float32, np.int8)):
        x = tokens(rng, 9, width, x_type)
        w = None if w_type is None else rng.standard_normal(width).astype(w_type)
        b = None if w_type is None or pitch == 8 else rng.standard_normal(width).astype(w_type)
        check_forward(x, w, b, y_type, "%s %s" % (x_type, y_type), pitch=pitch, shift=shift, stats=pitch != 3)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 15, 16, 17, 64, 255, 1000, 4099, 70001])
def test_forward_rows(rows):
    rng = rng_of(3, rows)
    for width in (24, 384, 520):
        check_forward(tokens(rng, rows, width, np.float16), None, None, np.float16, "%d x %d" % (rows, width))


@pytest.mark.parametrize("width", [48, 384, 1000, 4096, 20000])
@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_forward_in_place(width, dtype):
    rng = rng_of(4, width)
    check_forward(tokens(rng, 7, width, dtype), None, None, dtype, "in place", pitch=2, in_place=True)


@pytest.mark.parametrize("y_type", [np.float32, np.int8])
@pytest.mark.parametrize("width", [5, 384, 1000, 5000, 20000])
def test_forward_values(width, y_type):
    """Rows far from zero, equal values, zeros, the largest and smallest, and rows with a NaN or an infinity."""
    rng = rng_of(5, width)
    x = tokens(rng, 12, width, np.float32)
    x[0] += 5000.0
    x[1] = 3.25
    x[2] = 0.0
    x[3] *= 1e30
    x[4] *= 1e-30
    x[5, width // 2] = np.nan
    x[6, 0] = np.inf
    x[7, width - 1] = -np.inf
    x[8, 0] = 1e6                              # the value that the sums are taken from stands out
    x[9] = 1e8 + 64 * rng.integers(0, 2, width)
    check_forward(x, rng.standard_normal(width).astype(np.float32), rng.standard_normal(width).astype(np.float32), y_type, "values")


def test_forward_of_equal_values_without_eps():
    x = np.full((3, 100), 2.5, np.float16)
    got, stats, _ = forward(x, None, None, np.float16, eps=0.0)
    assert np.isnan(got).all() and np.isinf(stats[:, 1]).all() and (stats[:, 0] == 2.5).all()


def backward(x, gy, w, mean, rstd, want=("gx", "gweight", "gbias"), pitch=0, shift=0, w_type=np.float32, in_place=None):
    rows, width = x.shape
    xd, _ = placed(x, width + pitch, shift)
    gd, _ = placed(gy, width + pitch, shift)
    out = {}
    if "gx" in want:
        out["gx"] = {"x": xd, "gy": gd, None: placed(np.full((rows, width), 77, dtype=x.dtype), width + pitch, shift)[0]}[in_place]
    for name in ("gweight", "gbias"):
        if name in want:
            out[name] = torch.full((width,), 77.0, device="cuda", dtype=torch.float16 if w_type == np.float16 else torch.float32)
    stats = H.dev(np.stack([mean, rstd], 1).astype(np.float32))
    d = fq.FqNorm.from_torch(xd, weight=None if w is None else H.dev(w), stats=stats, gy=gd, **out)
    ws = torch.full((fq.fq_norm_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    fq.fq_norm_backward(d, ws)
    torch.cuda.synchronize()
    return {name: t.cpu().numpy() for name, t in out.items()}


def check_backward(x, gy, w, label, w_type=np.float32, **kw):
    with np.errstate(all="ignore"):
        _, _, mean, rstd = R.norm(x, None, None, EPS)
        mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    got = backward(x, gy, w, mean, rstd, w_type=w_type, **kw)
    want = R.norm_backward(x, gy, w, mean, rstd)
    for name, g in got.items():
        y, off = want[name]
        R.check(g, y, off, g.dtype == np.float16, "%s %s" % (label, name))


@pytest.mark.parametrize("g_type", [np.float16, np.float32])
@pytest.mark.parametrize("x_type", [np.float16, np.float32])
@pytest.mark.parametrize("width", WIDTHS + WIDE)
def test_backward_widths(width, x_type, g_type):
    rng = rng_of(6, width, x_type().itemsize, g_type().itemsize)
    for rows in (1, 5, 67):
        x, gy = tokens(rng, rows, width, x_type), tokens(rng, rows, width, g_type)
        check_backward(x, gy, (1 + 0.2 * rng.standard_normal(width)).astype(np.float32), "%d x %d" % (rows, width))


@pytest.mark.parametrize("rows,width", [(4099, 24), (70001, 24), (140000, 8), (19200, 384), (3001, 520), (2100, 4096), (1300, 20000)])
def test_backward_many_rows(rows, width):
    rng = rng_of(7, rows, width)
    x, gy = tokens(rng, rows, width, np.float16), tokens(rng, rows, width, np.float16)
    check_backward(x, gy, None, "%d x %d" % (rows, width))


@pytest.mark.parametrize("width,pitch,shift", [(40, 0, 1), (40, 1, 0), (384, 8, 8), (1155, 0, 3), (4096, 1, 1), (20000, 7, 1)])
def test_backward_strides_types_and_parts(width, pitch, shift):
    rng = rng_of(8, width, pitch)
    x, gy = tokens(rng, 37, width, np.float16), tokens(rng, 37, width, np.float16)
    w = rng.standard_normal(width).astype(np.float16)
    for want in (("gx", "gweight", "gbias"), ("gx",), ("gweight",), ("gbias", "gx"), ("gweight", "gbias")):
        check_backward(x, gy, w, str(want), w_type=np.float16, want=want, pitch=pitch, shift=shift)
    for in_place in ("x", "gy"):
        check_backward(x, gy, w, in_place, w_type=np.float16, pitch=pitch, shift=shift, in_place=in_place)


def test_backward_without_rows_gives_zeros():
    for dtype in (np.float16, np.float32):
        z = np.zeros((0, 300), np.float16)
        got = backward(z, z, None, np.zeros(0), np.zeros(0), w_type=dtype)
        assert (got["gweight"] == 0).all() and (got["gbias"] == 0).all() and got["gx"].shape == (0, 300)


@pytest.mark.parametrize("width", [384, 1000, 4096, 20000])
def test_backward_keeps_a_bad_row_to_itself(width):
    """A NaN in a row makes that row of gx NaN and the columns it is in; other rows are as they are without it."""
    rng = rng_of(9, width)
    x, gy = tokens(rng, 21, width, np.float32), tokens(rng, 21, width, np.float32)
    _, _, mean, rstd = R.norm(x, None, None, EPS)
    good = backward(x, gy, None, mean, rstd)
    gy[4, 3] = np.nan
    bad = backward(x, gy, None, mean, rstd)
    others = np.arange(21) != 4
    assert np.isnan(bad["gx"][4]).all() and np.array_equal(bad["gx"][others], good["gx"][others])
    columns = np.arange(width) != 3
    for name in ("gweight", "gbias"):
        assert np.isnan(bad[name][3]) and np.array_equal(bad[name][columns], good[name][columns])


@pytest.mark.parametrize("width", [40, 384, 1000, 4096])
def test_gradients_against_differences(width):
    """Central differences of sum(y * gy) in 64 bits along random directions: within their h^2 and the gradients' own tolerance."""
    rng = rng_of(10, width)
    x, gy = tokens(rng, 6, width, np.float32), tokens(rng, 6, width, np.float32)
    w, b = rng.standard_normal(width).astype(np.float32), rng.standard_normal(width).astype(np.float32)
    _, _, mean, rstd = R.norm(x, w, b, EPS)
    got = backward(x, gy, w, mean, rstd)
    loss = lambda x, w, b: (R.norm(x, w, b, EPS)[0] * gy.astype(np.float64)).sum()     # noqa: E731
    for name, at in (("gx", 0), ("gweight", 1), ("gbias", 2)):
        args = [x.astype(np.float64), w.astype(np.float64), b.astype(np.float64)]
        v = rng.standard_normal(args[at].shape)
        v /= np.linalg.norm(v)
        h, sides = 1e-4, []
        for sign in (1, -1):
            moved = list(args)
            moved[at] = args[at] + sign * h * v
            sides.append(loss(*moved))
        want = (sides[0] - sides[1]) / (2 * h)
        # third derivatives are of the order rstd^3 |gy| |v|^3: h^2 of it, and the binary32 of the gradient
        assert abs((got[name].astype(np.float64) * v).sum() - want) <= 1e-5 * np.linalg.norm(got[name].astype(np.float64)) + 1e-7 * np.abs(gy).sum() * h


def test_same_bits_every_time_and_captured():
    """A captured pass, replayed with the program's own work between, gives the bits of the eager one on other inputs, too."""
    torch.manual_seed(0)
    x, gy = torch.randn(3001, 384, device="cuda", dtype=torch.float16), torch.randn(3001, 384, device="cuda", dtype=torch.float16)
    w, b = torch.randn(384, device="cuda"), torch.randn(384, device="cuda")
    y, gx, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(3001, 2, device="cuda")
    gw, gb = torch.empty_like(w), torch.empty_like(b)
    q, ys = torch.empty(3001, 384, device="cuda", dtype=torch.int8), torch.empty(3001, device="cuda")
    d = fq.FqNorm.from_torch(x, y=y, weight=w, bias=b, stats=stats, gy=gy, gx=gx, gweight=gw, gbias=gb)
    c = fq.FqNorm.from_torch(x, y=q, weight=w, bias=b, y_scale=ys)
    ws = torch.empty(fq.fq_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    def work():
        fq.fq_norm_forward(d)
        fq.fq_norm_forward(c)
        fq.fq_norm_backward(d, ws)
    work()
    outs = (y, stats, gx, gw, gb, q, ys)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work()
    for seed in range(4):
        torch.manual_seed(seed)
        x.normal_()
        gy.normal_()
        work()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        ws.fill_(0xEE)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, v in zip(outs, want):
            assert torch.equal(t, v)

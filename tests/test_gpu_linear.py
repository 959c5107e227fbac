"""fq_linear_forward against the plain implementation in 64 bits: types, sizes off every grid, pitches, alignments, rows
that are zero or not finite, empty extents, streams, graphs, and that nothing outside the operands is read or written."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq
from paper_2511_12653_amd import workloads

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu

TORCH = {"f16": torch.float16, "f32": torch.float32, "i8": torch.int8}
NUMPY = {"f16": np.float16, "f32": np.float32, "i8": np.int8}


class Buffer:
    """A matrix on the GPU whose rows lie `pitch` elements apart, `front` elements behind the buffer's begin; all else
    in the buffer keeps a pattern."""

    def __init__(self, rows, cols, kind, pitch=None, front=0, values=None):
        self.pitch = cols if pitch is None else pitch
        self.fill = {"i8": 93, "f16": -24576.0, "f32": -24576.0}[kind]
        self.whole = torch.full((front + max(0, rows - 1) * self.pitch + cols + 40,), self.fill, dtype=TORCH[kind], device="cuda")
        self.view = torch.as_strided(self.whole, (rows, cols), (self.pitch, 1), front)
        if values is not None:
            self.view.copy_(H.dev(values))

    def untouched_outside(self):
        mask = torch.ones_like(self.whole, dtype=torch.bool)
        torch.as_strided(mask, self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(False)
        return bool((self.whole[mask] == self.fill).all())


def inputs(rng, m, n, k, x_kind, bias, xs_one=False, ws_one=False, spread=1.0):
    w = rng.integers(-128, 128, (n, k)).astype(np.int8)
    ws = (rng.uniform(0.5, 2.0, 1 if ws_one else n) * 1e-3).astype(np.float32)
    b = rng.standard_normal(n).astype(np.float32) if bias else None
    if x_kind == "i8":
        return rng.integers(-128, 128, (m, k)).astype(np.int8), (rng.uniform(0.5, 2.0, 1 if xs_one else m) * 1e-2).astype(np.float32), w, ws, b
    x = (rng.standard_normal((m, k)) * spread * np.exp(rng.standard_normal((m, 1)))).astype(NUMPY[x_kind])
    return x, None, w, ws, b


def reference(x, xs, w, ws, b, half):
    n, m = w.shape[0], x.shape[0]
    q, s = (x.astype(np.int64), xs) if xs is not None else R.quantize_rows(x)
    return R.linear(q, np.broadcast_to(s, (m,)), w, np.broadcast_to(ws, (n,)), b, half)


def call(x, xs, w, ws, b, y_kind, x_pitch=None, w_pitch=None, y_pitch=None, fronts=(0, 0, 0), stream=None, label=""):
    m, n = x.shape[0], w.shape[0]
    x_kind = {np.dtype(np.float16): "f16", np.dtype(np.float32): "f32", np.dtype(np.int8): "i8"}[x.dtype]
    bx, bw = Buffer(m, x.shape[1], x_kind, x_pitch, fronts[0], x), Buffer(n, w.shape[1], "i8", w_pitch, fronts[1], w)
    by = Buffer(m, n, y_kind, y_pitch, fronts[2])
    put = lambda a: None if a is None else H.dev(a)      # noqa: E731
    d = fq.FqLinear.from_torch(bx.view, bw.view, put(ws), by.view, bias=put(b), x_scale=put(xs))
    nbytes = fq.fq_linear_workspace_bytes(d)
    assert nbytes >= 256
    ws_buffer = torch.full((nbytes + 256,), 0xA5, dtype=torch.uint8, device="cuda")     # not initialised, and a guard
    torch.cuda.synchronize()
    fq.fq_linear_forward(d, (ws_buffer.data_ptr(), nbytes), stream) if stream else fq.fq_linear_forward(d, (ws_buffer.data_ptr(), nbytes))
    torch.cuda.synchronize()
    assert bool((ws_buffer[nbytes:] == 0xA5).all()), label + ": wrote behind the workspace"
    assert by.untouched_outside(), label + ": wrote outside y"
    assert bx.untouched_outside() and bw.untouched_outside()
    return by.view.cpu().numpy()


def run(m, n, k, x_kind, y_kind, seed, bias=True, xs_one=False, ws_one=False, **kw):
    label = "linear %dx%dx%d %s->%s %s" % (m, n, k, x_kind, y_kind, kw)
    H.say(label)
    rng = np.random.Generator(np.random.Philox(seed))
    given = inputs(rng, m, n, k, x_kind, bias, xs_one, ws_one)
    got = call(*given, y_kind, label=label, **kw)
    y, off = reference(*given, y_kind == "f16")
    R.check_linear(got, y, off, y_kind == "f16", label)


SIZES = [(1, 1, 1), (1, 16, 64), (1, 4096, 512), (1, 1000, 1155), (2, 33, 17), (3, 257, 100), (7, 64, 4096), (16, 128, 256),
         (17, 130, 384), (20, 512, 1024), (31, 48, 63), (33, 16, 2048), (64, 64, 64), (65, 300, 127), (100, 31, 129),
         (128, 256, 128), (129, 257, 255), (200, 96, 3456), (255, 511, 40), (256, 256, 512), (300, 700, 130), (513, 384, 384),
         (16, 64, 4000), (15, 70, 4288), (2, 40, 30000), (64, 8200, 96), (30, 16400, 200), (5, 16385, 80), (1024, 16, 16), (1029, 130, 300), (1100, 300, 511), (1027, 512, 512), (1200, 700, 64), (4000, 33, 65),
         (1050, 385, 384), (1100, 120, 500), (9000, 40, 100), (8200, 250, 256), (1000, 130, 1155), (1201, 257, 1155), (2049, 129, 96), (700, 1100, 640)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("x_kind,y_kind", [("f16", "f16"), ("f32", "f32"), ("i8", "f16")])
def test_sizes(m, n, k, x_kind, y_kind):
    run(m, n, k, x_kind, y_kind, seed=m * 7919 + n * 31 + k)


@pytest.mark.parametrize("m,n,k", [(1419, 5415, 130), (3362, 2314, 256), (1671, 4647, 385), (5393, 1416, 513), (1420, 5478, 1155),
                                   (5002, 772, 130), (712, 5462, 256), (5029, 773, 385), (5488, 708, 513), (706, 5456, 1155),
                                   (1331, 5397, 130), (1288, 5379, 256), (1281, 5510, 385), (1282, 5498, 1030),
                                   (514, 5473, 385), (5479, 513, 513), (5455, 517, 650), (580, 4913, 1030),
                                   (4913, 265, 256), (554, 1259, 385), (1960, 267, 513), (2832, 146, 650),
                                   (694, 1511, 256), (533, 775, 650), (1931, 135, 1030), (2048, 2304, 1024)])
def test_tiles_of_every_size(m, n, k):
    """One to ten steps of each tile, with ends that fill none."""
    run(m, n, k, "f16" if (m + k) % 2 else "i8", "f32" if n % 2 else "f16", seed=m)


@pytest.mark.parametrize("m", [1, 3, 16])
@pytest.mark.parametrize("k", [1, 15, 16, 100, 111, 112, 113, 127, 224, 225, 895, 896, 897, 1000, 2047, 4001])
@pytest.mark.parametrize("x_kind", ["f16", "f32", "i8"])
def test_few_tokens_with_rows_off_the_grid(m, k, x_kind):
    """Rows of w and x that begin anywhere in 16 bytes, around the steps that such rows are cut into."""
    for front in range(0, 16, 5):
        run(m, 50, k, x_kind, "f32", seed=k + front, w_pitch=k + front % 3, x_pitch=k + front % 2, fronts=(front, front, 0))


@pytest.mark.parametrize("m", [1, 5, 40, 300])
@pytest.mark.parametrize("x_kind,y_kind", [("f16", "f32"), ("f32", "f16"), ("i8", "f32")])
def test_other_types_single_scales_and_no_bias(m, x_kind, y_kind):
    run(m, 200, 320, x_kind, y_kind, seed=m, bias=False, xs_one=True, ws_one=True)


@pytest.mark.parametrize("m,n,k", [(1, 200, 512), (9, 200, 512), (150, 260, 512), (600, 512, 512), (150, 260, 515)])
@pytest.mark.parametrize("x_pitch,w_pitch,y_pitch,fronts", [(528, 544, 300, (0, 0, 0)), (517, 533, 261, (1, 3, 1)),
                                                            (None, 533, None, (8, 16, 0)), (640, None, 777, (3, 1, 2))])
@pytest.mark.parametrize("x_kind", ["f16", "i8", "f32"])
def test_pitches_and_alignments(m, n, k, x_pitch, w_pitch, y_pitch, fronts, x_kind):
    add = lambda p, least: None if p is None else max(p, p + least)     # noqa: E731
    run(m, n, k, x_kind, "f16", seed=k, x_pitch=add(x_pitch, k - 512), w_pitch=add(w_pitch, k - 512),
        y_pitch=add(y_pitch, max(0, n - 200)), fronts=fronts)


@pytest.mark.parametrize("m,n", [(17, 3), (33, 300), (100, 1100), (260, 129)])
@pytest.mark.parametrize("k", [16, 17, 24, 31, 33, 63, 64, 127, 136, 200, 256, 257, 300, 384, 399, 500, 511, 512, 513])
@pytest.mark.parametrize("x_kind", ["f16", "f32"])
def test_short_rows_of_any_length(m, n, k, x_kind):
    """Short rows of x against rows of w that begin anywhere: on 16 bytes, on words, between them."""
    for front, more in ((0, 0), (4, 4), (7, 3)):
        run(m, n, k, x_kind, "f16", seed=k + front, w_pitch=k + more, x_pitch=k + more % 4, fronts=(front % 4, front, 0))


@pytest.mark.parametrize("m,n,k", [(1500, 40, 250), (1030, 200, 300), (1025, 513, 127), (3000, 30, 511), (8200, 200, 77), (1024, 1100, 203)])
@pytest.mark.parametrize("front", [0, 5])
def test_short_rows_of_many_tokens(m, n, k, front):
    run(m, n, k, "f16", "f32", seed=k + front, w_pitch=k + 4 * front, fronts=(0, front, front))


@pytest.mark.parametrize("m", [1, 5, 16, 17, 32, 33, 64, 100])
@pytest.mark.parametrize("k", [513, 1008, 2001, 9000, 12345, 20000])
@pytest.mark.parametrize("x_kind", ["f16", "i8"])
def test_few_tokens_with_long_rows(m, k, x_kind):
    """Rows of x that leave no room in LDS, and more tokens than a block takes; w on 16 bytes and anywhere."""
    for front, more in ((0, -k % 16), (6, 3)):
        run(m, 37, k, x_kind, "f32", seed=k + front, w_pitch=k + more, x_pitch=k + (more if x_kind == "i8" else 0), fronts=(front if x_kind == "i8" else 0, front, 0))


@pytest.mark.parametrize("m", [1, 15, 16, 17, 50])
@pytest.mark.parametrize("k", [1, 7, 15, 16, 17, 96, 111, 112, 113, 128, 225, 800])
@pytest.mark.parametrize("x_front,x_more,w_front,w_more", [(1, 1, 0, 0), (5, 3, 5, 3), (0, 13, 9, 0), (16, 0, 3, 2), (15, 16, 0, 16)])
def test_few_tokens_of_codes_at_any_address(m, k, x_front, x_more, w_front, w_more):
    run(m, 50, k, "i8", "f16", seed=k + m, x_pitch=k + x_more, w_pitch=k + w_more, fronts=(x_front, w_front, 0))


@pytest.mark.parametrize("m,n,k", [(3, 20, 131071), (20, 4096, 640), (20, 4090, 639), (257, 464, 520), (8190, 16, 530)])
@pytest.mark.parametrize("x_kind", ["f32", "i8"])
def test_the_most_blocks_of_few_tokens(m, n, k, x_kind):
    run(m, n, k, x_kind, "f16", seed=m + n)


def test_rows_of_y_in_the_gaps_of_x():
    """x and y as columns of one buffer."""
    rng = np.random.Generator(np.random.Philox(5))
    x, _, w, ws, b = inputs(rng, 40, 24, 96, "f16", True)
    both = torch.zeros((40, 128), dtype=torch.float16, device="cuda")
    both[:, 8:104] = H.dev(x)
    d = fq.FqLinear.from_torch(both[:, 8:104], H.dev(w), H.dev(ws), both[:, 104:], bias=H.dev(b))
    fq.fq_linear_forward(d, torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    y, off = reference(x, None, w, ws, b, True)
    R.check_linear(both[:, 104:].cpu().numpy(), y, off, True)
    assert np.array_equal(both[:, 8:104].cpu().numpy(), x) and bool((both[:, :8] == 0).all())


@pytest.mark.parametrize("m", [1, 6, 70, 400])
@pytest.mark.parametrize("x_kind", ["f16", "f32"])
def test_rows_without_values(m, x_kind):
    """Rows that are all zero, tiny, huge, one value, or hold a NaN or an infinity."""
    rng = np.random.Generator(np.random.Philox(m))
    k, n = 300, 130
    x, _, w, ws, b = inputs(rng, m, n, k, x_kind, True)
    kinds = ["zero", "tiny", "huge", "one", "nan", "inf", "-inf", "-0", "subnormal"]
    at = rng.permutation(max(m, len(kinds)))[:len(kinds)]
    for kind, i in zip(kinds, at):
        if i >= m:
            continue
        if kind in ("zero", "-0", "one", "subnormal"):
            x[i] = -0.0 if kind == "-0" else 0.0
        if kind == "one":
            x[i, 17] = -3.5
        elif kind == "tiny":
            x[i] = np.sign(x[i]) * (2.0 ** -24 if x_kind == "f16" else 1.4e-36)
        elif kind == "subnormal":
            x[i, ::3] = 2.0 ** -24 if x_kind == "f16" else 1e-40
        elif kind == "huge":
            x[i, 5] = 65504.0 if x_kind == "f16" else 3.0e38
        elif kind in ("nan", "inf", "-inf"):
            x[i, rng.integers(k)] = float(kind)
    got = call(x, None, w, ws, b, "f32", label="rows")
    y, off = reference(x, None, w, ws, b, False)
    R.check_linear(got, y, off, False, "rows %d %s" % (m, x_kind))


@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_halves_of_the_code_steps(kind):
    """Quotients on and next to the halves, where a wrong rounding of the quotient shows in the code: one value per
    column against a unit matrix, so y / scale is the code."""
    k = 256
    x = np.zeros((64, k), np.float32)
    rng = np.random.Generator(np.random.Philox(11))
    top = rng.uniform(0.1, 50.0, 64)
    x[:, :254] = (np.arange(254) // 2 - 63 + 0.5)[None, :] * (top / 127)[:, None]
    x[:, 0] = top
    x = x.astype(NUMPY[kind])
    if kind == "f32":                                  # one unit up and down
        x[:, 1:128] = np.nextafter(x[:, 1:128], np.float32(np.inf))
        x[:, 128:254] = np.nextafter(x[:, 128:254], np.float32(-np.inf))
    w = np.eye(k, dtype=np.int8)
    got = call(x, None, w, np.ones(1, np.float32), None, "f32", label="halves")
    q, s = R.quantize_rows(x)
    assert np.array_equal(got, (q.astype(np.float32) * s[:, None]))


def test_largest_sums():
    """k at its limit with codes of the largest magnitude: the sum is just under 2^31."""
    k = 131071
    x, w = np.full((2, k), -128, np.int8), np.full((3, k), -128, np.int8)
    x[1], w[1] = 127, 127
    given = (x, np.array([1.0], np.float32), w, np.array([1.0], np.float32), None)
    y, off = reference(*given, False)
    R.check_linear(call(*given, "f32", label="largest"), y, off, False)
    rng = np.random.Generator(np.random.Philox(9))
    given = inputs(rng, 70, 40, k, "f16", True)
    y, off = reference(*given, False)
    R.check_linear(call(*given, "f32", label="longest rows"), y, off, False)


@pytest.mark.parametrize("m,n,k", [(0, 5, 7), (5, 0, 7), (5, 7, 0), (300, 20, 0), (0, 0, 0)])
@pytest.mark.parametrize("x_kind", ["f16", "i8"])
def test_empty_extents(m, n, k, x_kind):
    rng = np.random.Generator(np.random.Philox(3))
    x = np.zeros((m, k), NUMPY[x_kind])
    xs = np.full(max(1, m), 0.5, np.float32)[:m] if x_kind == "i8" else None
    if x_kind == "i8" and m == 0:
        xs = np.zeros(0, np.float32)
    w, ws, b = np.zeros((n, k), np.int8), np.ones(n, np.float32), rng.standard_normal(n).astype(np.float32)
    got = call(x, xs, w, ws, b, "f32", label="empty")
    assert np.array_equal(got, np.broadcast_to(b, (m, n)))


def test_codes_of_fq_forward_give_the_fake_quantized_product():
    """The codes and scales that fq_forward writes for a weight and an activation, multiplied here, against the product
    of the fake-quantized tensors in 64 bits."""
    rng = np.random.Generator(np.random.Philox(21))
    m, n, k = 300, 96, 200
    x, w = rng.standard_normal((m, k)).astype(np.float32), (rng.standard_normal((n, k)) * 0.1).astype(np.float32)
    th_x = workloads.theta_for_scale(np.array([4.0 / 127]))
    th_w = workloads.theta_for_scale(np.abs(w).max(axis=1) / 127)
    got = {}
    for name, a, theta, outer, channels, inner in (("x", x, th_x, 1, 1, m * k), ("w", w, th_w, 1, n, k)):
        ad, td = H.dev(a), H.dev(theta)
        q, s, y = torch.empty(a.shape, dtype=torch.int8, device="cuda"), torch.empty(channels, device="cuda"), torch.empty_like(ad)
        fq.fq_forward(fq.FqTensor.from_torch(outer, channels, inner, -127, 127, x=ad, y=y, q=q, theta=td, s=s))
        torch.cuda.synchronize()
        got[name] = (q, s, y.double().cpu().numpy())
    y = torch.empty((m, n), device="cuda")
    d = fq.FqLinear.from_torch(got["x"][0], got["w"][0], got["w"][1], y, x_scale=got["x"][1])
    fq.fq_linear_forward(d, torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    want = got["x"][2] @ got["w"][2].T
    # the fake-quantized values are rounded once each (2^-24), the product four times
    bound = 2.0 ** -24 * (2 * np.abs(got["x"][2]) @ np.abs(got["w"][2]).T + 5 * np.abs(want))
    assert np.all(np.abs(y.cpu().numpy() - want) <= bound)


@pytest.mark.parametrize("m,n,k", [(1, 512, 768), (20, 300, 640), (150, 384, 384), (700, 512, 1024)])
def test_graph_streams_and_repetition(m, n, k):
    """The same bits eagerly, on another stream, and in every replay of a graph, with other work in between."""
    rng = np.random.Generator(np.random.Philox(m))
    x, _, w, ws, b = inputs(rng, m, n, k, "f16", True)
    xd, wd, wsd, bd = (H.dev(a) for a in (x, w, ws, b))
    y = torch.empty((m, n), dtype=torch.float16, device="cuda")
    d = fq.FqLinear.from_torch(xd, wd, wsd, y, bias=bd)
    work = torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    fq.fq_linear_forward(d, work)
    first = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        fq.fq_linear_forward(d, work)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, first)
    y.zero_()
    fq.fq_linear_forward(d, work, torch.cuda.current_stream())
    assert torch.equal(y, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.fq_linear_forward(d, work)
    other = H.dev(inputs(rng, m, n, k, "f16", True)[0])
    for turn in range(6):
        y.fill_(7.0)
        work.fill_(turn * 37 % 251)
        xd.copy_(other if turn % 2 else H.dev(x))
        graph.replay()
        torch.cuda.synchronize()
        if turn % 2 == 0:
            assert torch.equal(y, first), "replay %d" % turn
        else:
            assert not torch.equal(y, first)

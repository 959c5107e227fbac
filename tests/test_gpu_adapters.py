"""fq_adapters_forward against the plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _more_operators_ref as R

pytestmark = pytest.mark.gpu


def case(m, k, n, count, rank, x_type, base_type, seed, order="mixed"):
    rng = np.random.Generator(np.random.Philox(seed))
    x = rng.standard_normal((m, k)) * np.exp(0.5 * rng.standard_normal((m, 1)))
    xs = None
    if x_type == np.int8:
        xs = (np.abs(x).max(1, initial=1e-3) / 127).astype(np.float32)
        x = np.clip(np.rint(x / xs[:, None]), -127, 127)
    ids = rng.integers(-1, count + 1, m) if count else np.full(m, 0)        # (-1 and count: none)
    if order == "runs":
        ids = np.sort(ids)
    return dict(x=x.astype(x_type), x_scale=xs, ids=ids.astype(np.int32), a=(rng.standard_normal((count, rank, k)) / np.sqrt(max(1, k))).astype(np.float16),
                b=(rng.standard_normal((count, n, rank)) / np.sqrt(max(1, rank))).astype(np.float16), scale=rng.uniform(0.5, 2, count).astype(np.float32),
                base=None if base_type is None else rng.standard_normal((m, n)).astype(base_type))


def placed(a, pitch, shift):
    rows, width = a.shape
    flat = torch.full((shift + max(1, rows) * (width + pitch),), 99, dtype=H.dev(a[:0]).dtype, device="cuda")
    view = flat[shift:shift + rows * (width + pitch)].view(rows, width + pitch)[:, :width]
    view.copy_(H.dev(a))
    return view, flat


def shifted(a, shift):
    """A contiguous copy that begins `shift` elements behind an allocation's begin."""
    flat = torch.empty(a.size + shift, dtype=H.dev(a.reshape(-1)[:0]).dtype, device="cuda")
    view = flat[shift:].view(a.shape)
    view.copy_(H.dev(a))
    return view


def run(c, y_type, pitch=0, shift=0, in_place=False):
    m, n = c["x"].shape[0], c["b"].shape[1]
    x, _ = placed(c["x"], pitch, shift)
    base = None if c["base"] is None else placed(c["base"], pitch, shift)[0]
    if in_place:
        y, flat = base, base
    else:
        y, flat = placed(np.full((m, n), 77, dtype=y_type), pitch, shift)
    dev = lambda name: None if c[name] is None else H.dev(c[name])     # noqa: E731
    d = fq.FqAdapters.from_torch(x, dev("ids"), shifted(c["a"], shift), shifted(c["b"], shift), y, base=base, scale=dev("scale"), x_scale=dev("x_scale"))
    ws = torch.full((fq.fq_adapters_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device="cuda")
    fq.fq_adapters_forward(d, ws)
    torch.cuda.synchronize()
    if pitch and not in_place:
        assert (flat.cpu().numpy()[shift:].reshape(m, n + pitch)[:, n:] == 99).all()
    return y.cpu().numpy()


def check(c, y_type, label="", **kw):
    got = run(c, y_type, **kw)
    y, off = R.adapters(**c)
    R.check(got, y, off, y_type == np.float16, label)
    none = (c["ids"] < 0) | (c["ids"] >= c["a"].shape[0])          # these are the base itself
    if c["base"] is not None and c["base"].dtype == y_type:
        assert np.array_equal(got[none], c["base"][none])


@pytest.mark.parametrize("x_type", [np.float16, np.float32, np.int8])
@pytest.mark.parametrize("m", [1, 2, 3, 15, 16, 17, 48, 64, 65, 129, 300])
def test_tokens(m, x_type):
    for order in ("mixed", "runs"):
        for count in (1, 3, 40):
            check(case(m, 264, 136, count, 16, x_type, np.float16, m * 10 + count, order), np.float16, "%s %d" % (order, count))


@pytest.mark.parametrize("rank", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 24, 31, 32, 33, 48, 63, 64, 65, 100, 128, 200, 256])
def test_ranks(rank):
    for m, x_type in ((1, np.float16), (5, np.int8), (70, np.float16), (33, np.float32)):
        check(case(m, 200, 120, 3, rank, x_type, np.float32, rank + m), np.float32, "%d" % m)


@pytest.mark.parametrize("k", [1, 2, 7, 8, 15, 16, 31, 32, 33, 63, 64, 65, 127, 255, 257, 512, 1000, 2047, 4096, 5001])
def test_values_per_token(k):
    for m, x_type in ((1, np.float16), (20, np.int8), (70, np.float16), (70, np.float32), (200, np.int8)):
        check(case(m, k, 72, 4, 12, x_type, np.float16, k + m), np.float16, "%d" % m)


@pytest.mark.parametrize("n", [1, 2, 7, 8, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 4097])
def test_channels(n):
    for m, y_type in ((1, np.float16), (20, np.float32), (70, np.float16), (130, np.float32)):
        check(case(m, 96, n, 4, 20, np.float16, np.float32 if m == 70 else np.float16, n + m), y_type, "%d" % m)


@pytest.mark.parametrize("pitch,shift", [(0, 1), (1, 0), (3, 5), (8, 8), (16, 16)])
def test_strides(pitch, shift):
    for m, k, n, rank, x_type in ((3, 128, 64, 8, np.float16), (40, 77, 99, 5, np.float16), (100, 264, 200, 16, np.int8), (90, 256, 128, 33, np.float32)):
        for y_type in (np.float16, np.float32):
            check(case(m, k, n, 3, rank, x_type, np.float16, pitch + m), y_type, "%d" % m, pitch=pitch, shift=shift)


@pytest.mark.parametrize("y_type", [np.float16, np.float32])
@pytest.mark.parametrize("base_type", [None, np.float16, np.float32])
def test_base_and_scale(base_type, y_type):
    for m in (2, 100):
        c = case(m, 128, 80, 5, 16, np.float16, base_type, m)
        check(c, y_type)
        check(dict(c, scale=None), y_type)
        if base_type == y_type:
            check(c, y_type, in_place=True, pitch=3)
    c = case(30, 128, 80, 5, 16, np.int8, base_type, 3)
    check(dict(c, x_scale=c["x_scale"][:1]), y_type)


def test_no_adapters():
    for count, rank, k in ((0, 16, 64), (3, 0, 64), (3, 16, 0), (0, 0, 0)):
        for base_type in (np.float16, None):
            c = case(20, k, 50, count, rank, np.float16, base_type, 1)
            check(c, np.float16)


def test_empty():
    for m, n in ((0, 10), (10, 0)):
        assert run(case(m, 16, n, 2, 4, np.float16, np.float16, 1), np.float16).shape == (m, n)


def test_ids_of_any_value():
    c = case(64, 128, 64, 4, 8, np.float16, np.float16, 2)
    c["ids"][:] = np.tile(np.array([0, -1, 3, 4, 2 ** 31 - 1, -2 ** 31, 1, 2], np.int32), 8)
    check(c, np.float16)


def test_a_bad_token_or_adapter_stays_with_itself():
    for m in (4, 100):
        c = case(m, 256, 96, 3, 16, np.float16, np.float16, 5)
        c["ids"] = (np.arange(m) % 3).astype(np.int32)
        good = run(c, np.float16)
        c["x"][1, 7] = np.nan
        c["a"][2, 3, 9] = np.inf
        got = run(c, np.float16)
        fine = (c["ids"] != 2) & (np.arange(m) != 1)
        assert np.array_equal(got[fine], good[fine])
        assert np.isnan(got[1]).all() and not np.isfinite(got[c["ids"] == 2]).any()


def test_large_and_small_products():
    """x a^T beyond FP16's range, and far below its least."""
    for factor_a, factor_b, x_type in ((1.0, 2.0 ** -12, np.float32), (2.0 ** -10, 1.0, np.float32), (8.0, 2.0 ** -10, np.float16), (2.0 ** -12, 8.0, np.float16)):
        for m in (3, 80):
            c = case(m, 512, 100, 3, 24, x_type, np.float32, m)
            c["x"] = (c["x"].astype(np.float64) * {np.float32: 2.0 ** 30, np.float16: 2.0 ** 10}[x_type] ** (1 if factor_a >= 1 else -1)).astype(x_type)
            c["a"] = (c["a"] * np.float16(factor_a)).astype(np.float16)
            c["b"] = (c["b"] * np.float16(factor_b)).astype(np.float16)
            check(c, np.float32, "%g %d" % (factor_a, m))


def test_captured():
    c = case(77, 256, 200, 5, 16, np.float16, np.float16, 9)
    x, ids, a, b, base = (H.dev(c[n]) for n in ("x", "ids", "a", "b", "base"))
    y = torch.empty_like(base)
    d = fq.FqAdapters.from_torch(x, ids, a, b, y, base=base)
    ws = torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    fq.fq_adapters_forward(d, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fq.fq_adapters_forward(d, ws)
    for seed in range(4):
        torch.manual_seed(seed)
        x.normal_()
        ids.copy_(torch.randint(-1, 6, (77,), device="cuda"))
        fq.fq_adapters_forward(d, ws)
        want = y.clone()
        y.fill_(7)
        ws.fill_(0xEE)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)

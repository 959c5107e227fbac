"""fq_adapters_forward with more tokens than a block sorts out by itself, with many adapters, with places beyond 32 bits, and with values
that FP16 holds as subnormal numbers; against the plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _more_operators_ref as R
from test_gpu_adapters import case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x_type", [np.float16, np.float32, np.int8])
@pytest.mark.parametrize("m", [1023, 1024, 1025, 1100, 2049, 4095, 4096, 4097, 4103])
def test_tokens(m, x_type):
    for order, count, rank, k, n in (("runs", 3, 16, 128, 70), ("mixed", 5, 24, 72, 136), ("mixed", 61, 40, 64, 66), ("runs", 2, 64, 256, 129), ("mixed", 1, 100, 80, 40)):
        check(case(m, k, n, count, rank, x_type, np.float16, m + rank, order), np.float16, "%s %d adapters of %d" % (order, count, rank))


@pytest.mark.parametrize("rank", [1, 5, 8, 16, 17, 32, 33, 47, 64, 65, 130, 256])
def test_ranks(rank):
    for m, x_type, shift in ((1500, np.float16, 0), (1500, np.float16, 1), (2500, np.int8, 0), (4500, np.int8, 0), (4500, np.float32, 0)):
        check(case(m, 96, 48, 7, rank, x_type, np.float32, rank, "runs" if rank % 2 else "mixed"), np.float32, "%d %d" % (m, shift), shift=shift)


@pytest.mark.parametrize("n", [1, 2, 3, 5, 63, 64, 65, 200, 1030])
def test_channels(n):
    for rank, pitch in ((4, 1), (16, 0), (48, 3)):
        check(case(4200, 32, n, 4, rank, np.float16, np.float16, n + rank), np.float16, "%d" % rank, pitch=pitch)


@pytest.mark.parametrize("k", [1, 8, 15, 16, 17, 40, 1000])
def test_values_per_token(k):
    for m, x_type in ((1300, np.float16), (4096, np.int8), (4200, np.int8)):
        check(case(m, k, 24, 4, 36, x_type, np.float16, k), np.float16, "%d" % m)


@pytest.mark.parametrize("count", [1, 2, 15, 16, 63, 64, 65, 255, 1000, 1023, 1024, 1025, 3000])
def test_adapters(count):
    for m in (50, 900, 1300, 4096, 4133):
        check(case(m, 48, 40, count, 8, np.float16, np.float16, count + m), np.float16, "%d" % m)


def test_all_of_one_or_of_none():
    for m in (1024, 1025, 4096, 5000):
        c = case(m, 64, 32, 6, 16, np.float16, np.float16, m)
        for one in (0, 5, 6, -1):
            c["ids"][:] = one
            check(c, np.float16, "%d" % one)
        c["ids"][m // 2] = 2
        check(c, np.float16)


@pytest.mark.parametrize("m", [65535, 65536, 65537, 140001])
def test_calls_that_go_in_parts(m):
    check(case(m, 24, 16, 5, 8, np.int8 if m % 2 else np.float16, np.float16, m, "mixed" if m < 100000 else "runs"), np.float16)


@pytest.mark.parametrize("rest,count", [(100, 1000), (3000, 1000), (4097, 700), (20000, 1024), (700, 2000)])
def test_the_last_part_is_cut_up_otherwise(rest, count):
    """The last tokens are found by another way than the first 65536, or in smaller tiles, and what is found has to fit as well."""
    check(case(65536 + rest, 24, 16, count, 8, np.float16, np.float16, rest), np.float16)


def test_in_place_and_without_base():
    for m in (1100, 5000):
        c = case(m, 64, 77, 5, 40, np.float16, np.float16, m)
        check(c, np.float16, in_place=True, pitch=3)
        check(dict(c, base=None), np.float16)
        check(dict(c, scale=None), np.float16)


def test_orders_stay_as_they_are():
    """Tokens keep their results whatever else comes with them, and calls give the same bits every time."""
    c = case(3000, 64, 48, 9, 16, np.float16, np.float16, 3)
    x, ids, a, b, base = (H.dev(c[n]) for n in ("x", "ids", "a", "b", "base"))

    def run(order):
        y = torch.empty_like(base)
        d = fq.FqAdapters.from_torch(x[order].contiguous(), ids[order].contiguous(), a, b, y, base=base[order].contiguous())
        fq.fq_adapters_forward(d, torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
        return y

    everything = torch.arange(3000, device="cuda")
    first = run(everything)
    for _ in range(3):
        assert torch.equal(run(everything), first)
    for seed in range(3):
        torch.manual_seed(seed)
        order = torch.randperm(3000, device="cuda")
        assert torch.equal(run(order), first[order])


@pytest.mark.parametrize("m,rank", [(3, 16), (80, 8), (1200, 24), (4200, 64)])
def test_subnormal_values(m, rank):
    """x, a and b one after the other below FP16's least normal number, 2^-14."""
    rng = np.random.Generator(np.random.Philox(m))
    for small in ("x", "a", "b"):
        c = case(m, 256, 64, 3, rank, np.float16, None, m)
        for name in ("x", "a", "b"):
            c[name] = np.sign(c[name]) * rng.integers(1, 900, c[name].shape) * 2.0 ** -24 if name == small else c[name].astype(np.float64) * 64
            c[name] = c[name].astype(np.float16)
        check(c, np.float32, small)


def test_places_beyond_32_bits():
    """Rows of x, base and y 2^20 elements apart, more than 4 GiB in all."""
    m, k, n, pitch = 2100, 64, 40, (1 << 20) + 8
    c = case(m, k, n, 4, 16, np.float16, np.float16, 1)
    wide = {name: torch.zeros((m, pitch), dtype=torch.float16, device="cuda") for name in ("x", "base", "y")}
    x, base, y = wide["x"][:, 8:8 + k], wide["base"][:, 16:16 + n], wide["y"][:, 24:24 + n]
    x.copy_(H.dev(c["x"]))
    base.copy_(H.dev(c["base"]))
    d = fq.FqAdapters.from_torch(x, H.dev(c["ids"]), H.dev(c["a"]), H.dev(c["b"]), y, base=base, scale=H.dev(c["scale"]))
    fq.fq_adapters_forward(d, torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    want, off = R.adapters(**c)
    R.check(y.cpu().numpy(), want, off, True)


def test_adapters_beyond_32_bits():
    """300 adapters of 64 x 2^17 values, 5 GB of each product's weights, of which the first, one and the last are used."""
    count, rank, size, used = 300, 64, 1 << 17, [0, 257, 299]
    weights = torch.zeros((count, rank * size), dtype=torch.float16, device="cuda")
    few = case(7, size, 16, 3, rank, np.float16, np.float16, 2)
    few["ids"] = np.array([0, 1, 2, 2, 1, 0, 2], np.int32)
    weights[used] = H.dev(few["a"].reshape(3, -1))
    ids = torch.tensor(used, device="cuda", dtype=torch.int32)[H.dev(few["ids"]).long()]
    b = torch.zeros((count, 16, rank), dtype=torch.float16, device="cuda")
    b[used] = H.dev(few["b"])
    few["scale"] = None
    base = H.dev(few["base"])
    y = torch.empty_like(base)
    d = fq.FqAdapters.from_torch(H.dev(few["x"]), ids, weights.view(count, rank, size), b, y, base=base)
    fq.fq_adapters_forward(d, torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    R.check(y.cpu().numpy(), *R.adapters(**few), True)

    few = case(7, 64, size, 3, rank, np.float16, np.float16, 3)
    few["ids"] = np.array([0, 1, 2, 2, 1, 0, 2], np.int32)
    weights.zero_()
    weights[used] = H.dev(few["b"].reshape(3, -1))
    a = torch.zeros((count, rank, 64), dtype=torch.float16, device="cuda")
    a[used] = H.dev(few["a"])
    few["scale"] = None
    base = H.dev(few["base"])
    y = torch.empty_like(base)
    d = fq.FqAdapters.from_torch(H.dev(few["x"]), ids, a, weights.view(count, size, rank), y, base=base)
    fq.fq_adapters_forward(d, torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda"))
    R.check(y.cpu().numpy(), *R.adapters(**few), True)


def test_widest():
    """2^20 values per token and 2^20 channels."""
    check(case(2, 1 << 20, 9, 2, 2, np.int8, np.float16, 4), np.float16)
    check(case(2, 9, 1 << 20, 2, 2, np.float16, np.float16, 5), np.float16)


@pytest.mark.parametrize("m", [2500, 6000])
def test_captured(m):
    """With the tokens' order found anew in each replay."""
    c = case(m, 64, 48, 9, 16, np.float16, np.float16, 9)
    x, ids, a, b, base = (H.dev(c[n]) for n in ("x", "ids", "a", "b", "base"))
    y = torch.empty_like(base)
    d = fq.FqAdapters.from_torch(x, ids, a, b, y, base=base)
    ws = torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    fq.fq_adapters_forward(d, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]                # (of one workspace, one after the other)
    for graph in graphs:
        with torch.cuda.graph(graph, stream=side):
            fq.fq_adapters_forward(d, ws)
    for seed in range(4):
        torch.manual_seed(seed)
        x.normal_()
        ids.copy_(torch.randint(-1, 10, (m,), device="cuda"))
        fq.fq_adapters_forward(d, ws)
        want = y.clone()
        for graph in graphs:
            y.fill_(7)
            ws.fill_(0xEE)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)

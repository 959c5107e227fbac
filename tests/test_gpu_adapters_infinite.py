"""fq_adapters_forward with infinities in the adapters: y is infinite, or NaN, where the formula says so and nowhere else, whatever the kernels load beside a
row's values or split them into; against the plain implementation in 64 bits."""
import numpy as np
import pytest

import _more_operators_ref as R
from test_gpu_adapters import case, run

pytestmark = pytest.mark.gpu
INF = np.float16(np.inf)


def check(c, label, **kw):
    got = run(c, np.float32, **kw)
    with np.errstate(all="ignore"):
        y, off = R.adapters(**c)
        R.check(got, y, off, False, label)               # (NaN in the same places; what is finite, within its bounds)
    assert np.isinf(y).any()
    assert np.array_equal(got[np.isinf(y)], y[np.isinf(y)]), label + ": infinities"
    assert np.isfinite(got[np.isfinite(y)]).all(), label


def put(c, name, places):
    """Infinities of both signs at places (adapter, row, value) of a or b."""
    for i, at in enumerate(places):
        c[name][at] = INF if i % 2 == 0 else -INF


SHAPES = [(3, 72, 40, 12), (3, 77, 66, 24), (3, 9, 10, 3), (40, 200, 130, 33), (70, 136, 70, 16), (90, 100, 50, 7), (1500, 72, 40, 5), (1500, 40, 70, 20),
          (4200, 72, 40, 40), (48, 72, 4100, 12), (30, 72, 9, 100), (30, 75, 12, 200), (20, 72, 1, 20), (5, 24, 3, 1)]


@pytest.mark.parametrize("x_type", [np.float16, np.float32, np.int8])
@pytest.mark.parametrize("m,k,n,rank", SHAPES)
def test_in_a(m, k, n, rank, x_type):
    """At the begin of a rank's values, at their end and between."""
    for place in (0, k - 1, k // 2, max(k - 9, 0)):
        c = case(m, k, n, 40 if m == 48 else 3, rank, x_type, np.float32, m + rank)
        put(c, "a", [(1, rank // 2, place), (2, rank - 1, place), (2, 0, place)][:3 if rank > 1 else 2])
        c["ids"][:3] = (0, 1, 2)
        check(c, "%d" % place, shift=place % 2)


@pytest.mark.parametrize("x_type", [np.float16, np.float32])
@pytest.mark.parametrize("m,k,n,rank", SHAPES)
def test_in_b(m, k, n, rank, x_type):
    """At the begin of a channel's values, at their end and between."""
    for place in (0, rank - 1, rank // 2, max(rank - 9, 0), min(8, rank - 1)):
        c = case(m, k, n, 40 if m == 48 else 3, rank, x_type, np.float16, m + rank)
        put(c, "b", [(1, 0, place), (1, n // 2, place), (2, n - 1, place)])
        c["ids"][:3] = (0, 1, 2)
        check(c, "%d" % place, shift=place % 2)


@pytest.mark.parametrize("m,k,n,rank", [s for s in SHAPES if s[3] > 1])
def test_beside_values_beyond_the_range_of_fp16(m, k, n, rank):
    """A token with one infinite t, and others of 2^20 and more."""
    c = case(m, k, n, 40 if m == 48 else 3, rank, np.float32, None, m + rank)
    c["x"] = (c["x"].astype(np.float64) * 2.0 ** 24).astype(np.float32)
    put(c, "a", [(1, 0, 0), (2, rank - 1, k - 1)])
    c["ids"][:3] = (0, 1, 2)
    check(c, "")


@pytest.mark.parametrize("m,k,n,rank", SHAPES)
def test_in_both(m, k, n, rank):
    c = case(m, k, n, 40 if m == 48 else 3, rank, np.float16, np.float32, m + rank)
    put(c, "a", [(1, rank // 2, 0), (2, 0, k - 1)])
    put(c, "b", [(1, 0, rank // 2), (0, n // 2, rank - 1), (2, n - 1, 0)])
    c["b"][2, n // 3, 0] = np.nan
    c["ids"][:3] = (0, 1, 2)
    check(c, "")


@pytest.mark.parametrize("m,k,n,rank", SHAPES)
def test_in_place_and_nan(m, k, n, rank):
    """y in place of base, infinities in some channels of b and NaN alone in others, each of which keeps to its channel."""
    c = case(m, k, n, 40 if m == 48 else 3, rank, np.float16, np.float32, m + rank)
    put(c, "b", [(1, n // 2, rank - 1)])
    c["b"][2, n // 3, 0] = np.nan
    c["b"][0, n - 1, rank // 2] = np.nan
    c["ids"][:3] = (0, 1, 2)
    check(c, "in place", in_place=True, pitch=3)

"""fq_adapters_forward near both ends of binary32's range, where a token's t, a scale or the power of two between them leaves it and y does not; against
the plain implementation in 64 bits, with its bounds as they are."""
import numpy as np
import pytest

import _more_operators_ref as R
from test_gpu_adapters import case, run

pytestmark = pytest.mark.gpu


def values(rng, shape, exponent, signs=True):
    """Of magnitude 2^exponent to 2^(exponent + 1)."""
    v = rng.uniform(1, 2, shape) * 2.0 ** exponent
    return v * rng.choice([-1.0, 1.0], shape) if signs else v


def check(c):
    got = run(c, np.float32)
    y, off = R.adapters(**c)
    R.check(got, y, off, False)
    held = np.isin(c["ids"], np.arange(c["a"].shape[0]))
    size = np.abs(y[held])
    assert ((size > 2.0 ** -126) & np.isfinite(size)).any()          # (something normal to be right about; b of 2^16, which FP16 lacks, makes some y infinite)


@pytest.mark.parametrize("m,n,rank", [(3, 100, 12), (80, 66, 24), (1500, 40, 5), (48, 4100, 7), (20, 70, 100), (20, 70, 200)])
@pytest.mark.parametrize("x,scale,b", [(-124, 0, 10), (-120, 3, -3), (-124, -2, 15), (-100, -40, 15), (118, 20, -24), (100, 38, -24), (122, 0, -14)])
def test_tokens_near_the_ends(m, n, rank, x, scale, b):
    """x a^T of 2^-122 and less, or of 2^120 and more (all of a's and x's values positive: no sum is less than its terms, and no product of x and a subnormal)."""
    rng = np.random.Generator(np.random.Philox(m + rank))
    c = case(m, 16, n, 40 if m == 48 else 3, rank, np.float32, None, rank)
    c["x"] = values(rng, c["x"].shape, x, signs=False).astype(np.float32)
    c["a"] = values(rng, c["a"].shape, -1, signs=False).astype(np.float16)
    with np.errstate(over="ignore"):
        c["b"] = values(rng, c["b"].shape, b).astype(np.float16)
    c["scale"] = values(rng, c["scale"].shape, scale).astype(np.float32)
    check(c)


@pytest.mark.parametrize("m,rank", [(5, 16), (100, 40)])
@pytest.mark.parametrize("xs,scale", [(-80, -60), (-126, 20), (100, 40), (126, -126)])
def test_scales_whose_product_leaves_the_range(m, rank, xs, scale):
    """Codes and b of a size that brings y back into it."""
    rng = np.random.Generator(np.random.Philox(m + rank))
    c = case(m, 64, 80, 3, rank, np.int8, None, rank)
    small = xs + scale > 0
    c["x"] = (np.abs(c["x"]) if small else 100 + np.abs(c["x"]) % 28).astype(np.int8)
    c["a"] = values(rng, c["a"].shape, -13 if small else 12, signs=False).astype(np.float16)
    c["b"] = values(rng, c["b"].shape, -24 if small else 14).astype(np.float16)
    c["x_scale"] = values(rng, c["x_scale"].shape, xs, signs=False).astype(np.float32)
    c["scale"] = values(rng, c["scale"].shape, scale).astype(np.float32)
    check(c)

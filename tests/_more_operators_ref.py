"""Plain numpy implementations of layer norm, dropout and the adapters, written from the formulas in include/fq.h: in 64 bits, with
the most that a right result may be off; what the definition fixes bit by bit (random bits, codes) in the arithmetic it names."""
import numpy as np

U32, U16 = 2.0 ** -24, 2.0 ** -11          # half a step of binary32 and of FP16, relative to the value
TINY16, TINY32 = 2.0 ** -25, 2.0 ** -150   # half a step of the subnormal ones


def rounding(y, half):
    """The most that rounding y to its type moves it."""
    return np.abs(y) * U16 + TINY16 if half else np.abs(y) * U32 + TINY32


def check(got, y, off, half, label=""):
    """got against y, that may be off by `off` before it is rounded to its type."""
    got = got.astype(np.float64)
    assert got.shape == y.shape, "%s: %s instead of %s" % (label, got.shape, y.shape)
    assert np.array_equal(np.isnan(got), np.isnan(y)), label + ": NaN in other places"
    edge = 65520.0 if half else 3.4e38
    with np.errstate(all="ignore"):
        sure = np.abs(y) > edge + off
        assert np.all(np.isinf(got[sure]) & (np.sign(got[sure]) == np.sign(y[sure]))), label + ": overflow"
        fine = np.abs(y) < edge - off
        far = (np.abs(got - y) - off - rounding(np.abs(y) + off, half))[fine]
    assert far.size == 0 or far.max() <= 0, "%s: off by %.3e more than rounding allows" % (label, far.max())


# ---------------------------------------------------------------------------------------------------------------- norm
def norm(x, w, b, eps):
    """(y, off, mean, rstd) in 64 bits.  off: what binary32 arithmetic behind binary64 sums may be away: of the mean's and
    rstd's rounding, the difference, the two products and the sum, each half a step of what it makes."""
    with np.errstate(all="ignore"):
        x = x.astype(np.float64)
        mean = x.mean(1, keepdims=True)
        d = x - mean
        rstd = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
        w = np.ones(x.shape[1]) if w is None else w.astype(np.float64)
        b = np.zeros(x.shape[1]) if b is None else b.astype(np.float64)
        y = d * rstd * w + b
        off = 5 * U32 * np.abs(d * rstd * w) + U32 * np.abs(y) + 1e-12 * np.abs(mean * rstd * w) + TINY32
    return y, off, mean[:, 0], rstd[:, 0]


def codes(x, w, b, eps):
    """(codes, scales, how near y / s is to a half): y in 64 bits, rounded to binary32, quantized as fq_linear quantizes rows."""
    y, _, _, _ = norm(x, w, b, eps)
    with np.errstate(all="ignore"):
        y = y.astype(np.float32)
        fine = np.isfinite(y).all(1)
        top = np.where(fine, np.abs(y).max(1), np.float32(0)).astype(np.float32)
        zero = top < np.float32(127) * np.float32(2.0 ** -126)
        s = np.where(fine, np.where(zero, np.float32(0), top / np.float32(127)), np.float32(np.nan)).astype(np.float32)
        q = np.clip(np.rint(y / s[:, None]), -127, 127)
        near = np.abs(np.abs(y.astype(np.float64) / s[:, None].astype(np.float64)) % 1.0 - 0.5)
    keep = (fine & ~zero)[:, None]
    return np.where(keep, q, 0).astype(np.int64), s, np.where(keep, near, 1.0)


def norm_backward(x, gy, w, mean, rstd, wide=False):
    """{name: (value, off)} of gx, gweight, gbias in 64 bits, from the statistics (float32) as they are.

    In binary32, per element: h = (x - mean) * rstd (2 roundings), a = gy * w (1), a * h (1); then the sums over a row of k values
    and over the rows.  A sum of n terms in order of which each partial sum is rounded is off by at most n U32 sum |terms|; rows are
    added 8 at a time in binary32, then in binary64, so by 8; columns up to 256 rows (a block's), over 4 (16) row groups."""
    k = x.shape[1]
    x, gy, mean, rstd = (t.astype(np.float64) for t in (x, gy, mean[:, None], rstd[:, None]))
    w = np.ones(k) if w is None else w.astype(np.float64)
    with np.errstate(all="ignore"):
        h = (x - mean) * rstd
        a = gy * w
        c1, c2 = a.sum(1, keepdims=True) / k, (a * h).sum(1, keepdims=True) / k
        gx = rstd * (a - c1 - h * c2)
        size1, size2 = np.abs(a).sum(1, keepdims=True) / k, np.abs(a * h).sum(1, keepdims=True) / k
        off1, off2 = 11 * U32 * size1, 14 * U32 * size2
        off = rstd * (U32 * np.abs(a) + off1 + 3 * U32 * (np.abs(a) + np.abs(c1)) + np.abs(h) * off2 + 8 * U32 * np.abs(h * c2)) + U32 * np.abs(gx)
        gw, gb = (gy * h).sum(0), gy.sum(0)
        terms = min(x.shape[0], 256) + 8
        offw = (terms + 3) * U32 * np.abs(gy * h).sum(0) + TINY32
        offb = terms * U32 * np.abs(gy).sum(0) + TINY32
    return {"gx": (gx, off + TINY32), "gweight": (gw, offw), "gbias": (gb, offb)}


# ------------------------------------------------------------------------------------------------------------- dropout
def keys(seed, step, high=0):
    m = (1 << 64) - 1
    k = (seed * 0x9E3779B97F4A7C15 + step * 0xD1B54A32D192ED03 + high * 0x8CB92BA72F3D8DD7) & m
    k = ((k ^ (k >> 32)) * 0x9E3779B97F4A7C15) & m
    k = ((k ^ (k >> 29)) * 0xD1B54A32D192ED03) & m
    return k >> 32, (k ^ (k >> 32)) & 0xFFFFFFFF


def random_bits(place, seed, step):
    """place: uint64 array, all with the same upper 32 bits.  31 bits of each."""
    first, second = keys(seed, step, int(place[0] >> np.uint64(32)) if place.size else 0)
    m = np.uint64(0xFFFFFFFF)
    h = ((place & m) * np.uint64(0x9E3779B1) + np.uint64(first)) & m
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x6A09E667)) & m
    h = (((h ^ (h >> np.uint64(15))) + np.uint64(second) & m) * np.uint64(0xBB67AE85)) & m
    return h >> np.uint64(1)


def keep(n, p, seed, step, begin=0):
    at = np.arange(n, dtype=np.uint64) + np.uint64(begin)
    return random_bits(at, seed, step) >= np.uint64(round(p * (1 << 31)))


def dropout(x, p, seed, step, residual, half):
    """The very values: binary32 operations, each rounded, then rounding to y's type."""
    with np.errstate(all="ignore"):
        scale = np.float32(0.0 if p == 1.0 else 1.0 / (1.0 - p))
        y = np.where(keep(x.size, p, seed, step), x.astype(np.float32).reshape(-1) * scale, np.float32(0.0)).astype(np.float32)
        if residual is not None:
            y = y + residual.astype(np.float32).reshape(-1)
        return y.astype(np.float16 if half else np.float32).reshape(x.shape)


# ------------------------------------------------------------------------------------------------------------ adapters
def adapters(x, x_scale, ids, a, b, scale, base):
    """(y, off).  off: x * a sums in binary32 (products exact for FP16 and codes; FP32: rounded), in any order, but with partial
    sums over at least eight lanes; t held in 21 bits or more beside the row's greatest; the second sum likewise; the products with the scales and
    the sum with the base."""
    m, k = x.shape
    count, rank, _ = a.shape
    n = b.shape[1]
    x = x.astype(np.float64)
    xs = np.ones((m, 1)) if x_scale is None else np.broadcast_to(x_scale.astype(np.float64).reshape(-1, 1), (m, 1))
    y = np.zeros((m, n)) if base is None else base.astype(np.float64).copy()
    off = U32 * np.abs(y)
    with np.errstate(all="ignore"):
        for i in range(m):
            if not 0 <= ids[i] < count:
                continue
            wa, wb = a[ids[i]].astype(np.float64), b[ids[i]].astype(np.float64)
            s = 1.0 if scale is None else float(scale[ids[i]])
            t = wa @ x[i] * xs[i]
            size = np.abs(wa) @ np.abs(x[i]) * xs[i]
            d = s * (wb @ t)
            t_off = (k / 8 + 16) * U32 * size + 3 * U32 * np.abs(t) + 2.0 ** -21 * np.abs(t).max(initial=0.0)
            off[i] += abs(s) * (np.abs(wb) @ t_off + (rank + 8) * U32 * (np.abs(wb) @ np.abs(t))) + 3 * U32 * np.abs(d) + U32 * np.abs(y[i] + d)
            y[i] += d
    return y, off + TINY32

"""Plain numpy implementations of the int8 linear layer and of the AdamW step, written from the formulas in include/fq.h:
the values that the definition fixes bit by bit (codes, scales, binary32 moments) in the arithmetic it names, everything
else in 64 bits."""
import numpy as np

FLT_MIN = np.float32(2.0 ** -126)
F32 = np.float32


# ------------------------------------------------------------------------------------------------------------ linear
def quantize_rows(x):
    """(codes, scales) of the rows of x."""
    with np.errstate(all="ignore"):
        x = x.astype(np.float32)
        top = np.abs(x).max(axis=1, initial=0.0).astype(np.float32)
        fine = np.isfinite(top) & ~np.isnan(x).any(axis=1)
        zero = fine & (top < F32(127) * FLT_MIN)
        s = np.where(fine, np.where(zero, F32(0), top / F32(127)), F32(np.nan)).astype(np.float32)
        q = np.clip(np.rint(x / s[:, None]), -127, 127)
        q = np.where((fine & ~zero)[:, None], q, 0)
    return q.astype(np.int64), s


def linear(q, xs, w, ws, bias, half):
    """(y in 64 bits, the most that a right y may be off): each of the conversion of the sum, the product of the scales,
    the product and the addition may round by half a unit in the last place; so may the conversion to FP16."""
    with np.errstate(all="ignore"):
        total = (q.astype(np.float64) @ w.astype(np.float64).T)          # exact: below 2^53
        product = total * xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :]
        y = product if bias is None else product + bias.astype(np.float64)[None, :]
        u = 2.0 ** -24
        off = 4 * u * np.abs(product) + 2 * u * np.abs(y) + 2.0 ** -148
        if half:
            off = off + 2.0 ** -11 * np.abs(y) + 2.0 ** -24
    return y, off


def check_linear(got, y, off, half, label=""):
    got = got.astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(y)), label + ": NaN in other places"
    if half:                                  # from 65520 on FP16 has infinity; at the edge either is right
        sure = np.abs(y) > 65520 + off
        assert np.all(np.isinf(got[sure]) & (np.sign(got[sure]) == np.sign(y[sure]))), label + ": overflow"
        fine = ~np.isnan(y) & (np.abs(y) < 65520 - off)
    else:
        fine = np.isfinite(y)
        assert np.array_equal(got[~fine & ~np.isnan(y)], y[~fine & ~np.isnan(y)]), label
    with np.errstate(all="ignore"):
        far = np.abs(got - y)[fine] - off[fine]
    assert far.size == 0 or far.max() <= 0, "%s: off by %.3e more than rounding allows" % (label, far.max())


# ------------------------------------------------------------------------------------------------------------- AdamW
BLOCK = 256


def key(seed, step):
    m = (1 << 64) - 1
    k = (seed * 0x9E3779B97F4A7C15 + step * 0xD1B54A32D192ED03) & m
    return ((k ^ (k >> 32)) * 0x9E3779B97F4A7C15 & m) >> 32


def random_bits(place, k):
    """place: uint64 array.  The 32 bits of each."""
    m = np.uint64(0xFFFFFFFF)
    x = (place * np.uint64(0x9E3779B1) + np.uint64(k)) & m
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & m
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & m
    return x ^ (x >> np.uint64(16))


def _blocks(a):
    n = -(-a.size // BLOCK) * BLOCK
    return np.concatenate([a, np.zeros(n - a.size, a.dtype)]).reshape(-1, BLOCK)


def scale_exponent(top, least, power=1):
    """The least e >= least with top <= (448 * 2^e)^power, by comparison."""
    e = np.full(top.shape, least, np.int64)
    with np.errstate(over="ignore"):
        for _ in range(400):
            low = top.astype(np.float64) > (448.0 * np.exp2(e.astype(np.float64))) ** power
            if not low.any():
                return e
            e = e + low
    raise AssertionError


def round_codes(a, bits):
    """The code below a (>= 0, in steps) + (bits + 1/2) / 2^16 steps, in 64 bits."""
    a = a.astype(np.float64)
    with np.errstate(divide="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(a)), -6.0) - 3.0)
    return np.floor(a / step + (bits.astype(np.float64) + 0.5) / 65536.0) * step


def _mul(a, b):
    return (a.astype(np.float32) * F32(b)).astype(np.float32)


def step(p, g, m, v, m_scale, v_scale, h, place, lr_scale=1.0, weight_decay=0.0, grad_scale=None):
    """One tensor.  p, g: float32 or float16 arrays, m, v: float32 arrays (FP8: the values of the codes).  Returns a
    dict: p and how far a right p may be off (64 bits), and of the states either the binary32 values or, for FP8, the
    codes' values (m), the lowest and highest that a right code may be (v) and both scales."""
    f8 = m_scale is not None
    b1, c1, b2, c2 = F32(h["beta1"]), F32(1 - h["beta1"]), F32(h["beta2"]), F32(1 - h["beta2"])
    n = p.size
    with np.errstate(all="ignore"):
        g = g.astype(np.float32)
        if grad_scale is not None:
            g = _mul(g, grad_scale)
        if f8:
            m = _blocks(m).astype(np.float32) * m_scale[:, None].astype(np.float32)
            r = _blocks(v).astype(np.float32) * v_scale[:, None].astype(np.float32)
            m, v = m.reshape(-1)[:n], (r * r).reshape(-1)[:n]
        m1 = _mul(m, b1) + _mul(g, c1)
        v1 = _mul(v, b2) + _mul(g, c2) * g
        fine = np.isfinite(v1)
        m1, v1 = np.where(fine, m1, m).astype(np.float32), np.where(fine, v1, v).astype(np.float32)
        root = np.sqrt(v1.astype(np.float64))
        lr = h["lr"] * lr_scale
        below = root / np.sqrt(1 - h["beta2"] ** h["step"]) + h["eps"]
        move = lr / (1 - h["beta1"] ** h["step"]) * (m1.astype(np.float64) / below)
        p0 = p.astype(np.float64)
        p1 = np.where(fine, p0 * (1 - lr * weight_decay) - move, p0)
        # binary32: the constants, root, quotient and products of `move`, 12 units in all at most; `keep` (two roundings:
        # its own and lr's within lr * decay), the product and the subtraction
        u = 2.0 ** -24
        off = 12 * 2 * u * np.abs(move) + 3 * u * np.abs(p0) + u * np.abs(p1) + 4 * u * abs(lr * weight_decay) * np.abs(p0) + 2.0 ** -148
    out = {"p": p1, "off": np.where(fine, off, 0.0), "m": m1, "v": v1}
    if p.dtype == np.float16:
        out["off"] = out["off"] + np.where(fine, 2.0 ** -11 * np.abs(p1) + 2.0 ** -25, 0.0)
    if not f8:
        return out
    at = np.arange(-(-n // BLOCK) * BLOCK, dtype=np.uint64)
    bits = random_bits((at + np.uint64(place)) & np.uint64(0xFFFFFFFF), key(h["seed"], h["step"])).reshape(-1, BLOCK)
    low, high = bits & np.uint64(0xFFFF), bits >> np.uint64(16)
    mb, vb = _blocks(m1), _blocks(v1)
    em, ev = scale_exponent(np.abs(mb).max(axis=1), -126), scale_exponent(vb.max(axis=1), -63, 2)
    down = lambda e: np.exp2(-e.astype(np.float64))[:, None]     # noqa: E731
    # below 2^-6 the binary32 sum a + 2^-6 may round: by 2^-30, a millionth of a step
    a = np.abs(mb) * down(em)
    a = np.where(a < 2.0 ** -6, (a.astype(np.float32) + F32(2.0 ** -6)).astype(np.float64) - 2.0 ** -6, a)
    out["m8"] = (round_codes(a, low) * np.where(np.signbit(mb), -1.0, 1.0)).reshape(-1)[:n]
    r = np.sqrt(vb.astype(np.float64)) * down(ev)
    slack = 2.0 ** -22
    for name, value in (("v8_least", r * (1 - slack) - 2.0 ** -29), ("v8_most", r * (1 + slack) + 2.0 ** -29)):
        code = round_codes(np.maximum(value, 0.0), high)
        code = np.where(vb > 0, np.maximum(code, 2.0 ** -9), 0.0)
        out[name] = np.minimum(code, 448.0).reshape(-1)[:n]
    # and the code of the binary32 root, which is the one to expect
    a = np.sqrt(vb).astype(np.float64) * down(ev)
    a = np.where(a < 2.0 ** -6, (a.astype(np.float32) + F32(2.0 ** -6)).astype(np.float64) - 2.0 ** -6, a)
    out["v8"] = np.where(vb > 0, np.maximum(round_codes(a, high), 2.0 ** -9), 0.0).reshape(-1)[:n]
    out["m_scale"], out["v_scale"] = np.exp2(em.astype(np.float64)), np.exp2(ev.astype(np.float64))
    return out

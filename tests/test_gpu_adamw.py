"""fq_adamw_step against the plain implementation in 64 bits: types, states in FP32 and FP8, sizes off every grid, many
tensors, alignments, gradients that are not finite, steps in a row, streams and graphs."""
import numpy as np
import pytest
import torch

from paper_2511_12653_amd import binding as fq

import _gpu_harness as H
import _operators_ref as R

pytestmark = pytest.mark.gpu

NP = {"f16": np.float16, "f32": np.float32}
GUARD = 64


class Guarded:
    """A tensor inside a buffer with a pattern in front of and behind it, `off` elements off the 256-byte grid."""

    def __init__(self, a, off=0, dtype=None):
        t = H.dev(a)
        if dtype is not None:
            t = t.to(dtype)
        raw = torch.full(((a.size + off + GUARD * 2) * t.element_size(),), 0x5B, dtype=torch.uint8, device="cuda")
        self.raw, self.at, self.n = raw.view(t.dtype), GUARD + off, a.size
        self.t = self.raw[self.at:self.at + self.n]
        self.t.copy_(t.reshape(-1))
        self.bytes, self.each = raw, t.element_size()

    def host(self):
        return self.t.float().cpu().numpy() if self.t.dtype == torch.float8_e4m3fn else self.t.cpu().numpy()

    def check(self, label):
        a, b = self.at * self.each, (self.at + self.n) * self.each
        assert bool((self.bytes[:a] == 0x5B).all()) and bool((self.bytes[b:] == 0x5B).all()), label + ": wrote outside"


class Tensor:
    def __init__(self, rng, n, p="f32", g="f32", f8=False, copy=False, lr_scale=1.0, decay=0.0, off=0, spread=1.0, fresh=False):
        self.n, self.f8, self.lr_scale, self.decay = n, f8, lr_scale, decay
        g_ = (rng.standard_normal(n) * spread).astype(NP[g])
        m_ = (rng.standard_normal(n) * 0.3 * spread).astype(np.float32) * (not fresh)
        v_ = np.square(rng.standard_normal(n) * spread).astype(np.float32) * (not fresh)
        self.p, self.g = Guarded((rng.standard_normal(n) * 0.1).astype(NP[p]), off), Guarded(g_, off)
        self.copy = Guarded(np.zeros(n, np.float16), off) if copy else None
        blocks = -(-n // 256)
        self.ms = self.vs = None
        if f8:
            e = [R.scale_exponent(np.abs(R._blocks(a)).max(axis=1), -126) if n else np.zeros(0, np.int64) for a in (m_, np.sqrt(v_))]
            scale = [np.exp2(k.astype(np.float64)).astype(np.float32) for k in e]
            code = [(R._blocks(a) / s[:, None]).reshape(-1)[:n] for a, s in zip((m_, np.sqrt(v_)), scale)]
            self.m, self.v = (Guarded(c.astype(np.float32), off, torch.float8_e4m3fn) for c in code)
            self.ms, self.vs = Guarded(scale[0]), Guarded(scale[1])
            assert self.ms.n == blocks
        else:
            self.m, self.v = Guarded(m_, off), Guarded(v_, off)

    def param(self):
        t = lambda x: None if x is None else x.t      # noqa: E731
        return fq.FqParam.from_torch(self.p.t, self.g.t, self.m.t, self.v.t, t(self.ms), t(self.vs), t(self.copy),
                                     lr_scale=self.lr_scale, weight_decay=self.decay)

    def all(self):
        return [x for x in (self.p, self.g, self.m, self.v, self.ms, self.vs, self.copy) if x is not None]

    def reference(self, h, place, grad_scale):
        host = lambda x: None if x is None else x.host()      # noqa: E731
        return R.step(self.p.host(), self.g.host(), self.m.host(), self.v.host(), host(self.ms), host(self.vs), h, place,
                      self.lr_scale, self.decay, grad_scale)

    def compare(self, want, label):
        for x in self.all():
            x.check(label)
        got = self.p.host().astype(np.float64)
        assert np.array_equal(np.isnan(got), np.isnan(want["p"])), label
        with np.errstate(all="ignore"):
            far = np.abs(got - want["p"]) - want["off"]
        assert not (far > 0).any(), "%s: p off by %.3e more than rounding allows" % (label, np.nanmax(far))
        if self.copy is not None:
            with np.errstate(over="ignore"):
                assert np.array_equal(self.copy.host(), self.p.host().astype(np.float16), equal_nan=True), label + ": copy"
        if not self.f8:
            assert np.array_equal(self.m.host(), want["m"], equal_nan=True), label + ": m"
            assert np.array_equal(self.v.host(), want["v"], equal_nan=True), label + ": v"
            return
        assert np.array_equal(self.ms.host(), want["m_scale"].astype(np.float32)), label + ": m_scale"
        assert np.array_equal(self.vs.host(), want["v_scale"].astype(np.float32)), label + ": v_scale"
        assert np.array_equal(self.m.host(), want["m8"].astype(np.float32)), label + ": m"
        v = self.v.host().astype(np.float64)
        assert np.all((v >= want["v8_least"]) & (v <= want["v8_most"])), label + ": v"


HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=7, seed=123456789012345)


def make_plan(tensors):
    params = [t.param() for t in tensors]
    nbytes = fq.fq_adamw_workspace_bytes(params)
    assert nbytes >= 256
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return fq.fq_adamw_create(params, ws), ws


def run(tensors, label, steps=1, grad_scale=None, **hyper):
    H.say("adamw " + label)
    h = dict(HYPER, **hyper)
    plan, ws = make_plan(tensors)
    gs = None if grad_scale is None else torch.tensor([grad_scale], dtype=torch.float32, device="cuda")
    hy = fq.FqAdamW(grad_scale=gs, **h)
    for i in range(steps):
        h["step"] = hy.step = HYPER["step"] + i
        want, place = [], 0
        for t in tensors:
            want.append(t.reference(h, place, None if grad_scale is None else np.float32(grad_scale)))
            place += -(-t.n // 256) * 256
        fq.fq_adamw_step(plan, hy)
        torch.cuda.synchronize()
        for k, (t, w) in enumerate(zip(tensors, want)):
            t.compare(w, "%s, step %d, tensor %d of %d elements" % (label, i, k, t.n))
    fq.fq_adamw_destroy(plan)


SIZES = [1, 2, 3, 4, 5, 63, 64, 255, 256, 257, 300, 511, 512, 1000, 1023, 1024, 1025, 2049, 4095, 4096, 4097, 5000, 70001]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("p,g,copy", [("f32", "f32", False), ("f32", "f16", True), ("f16", "f16", False), ("f16", "f32", False),
                                      ("f32", "f32", True)])
def test_types_and_sizes(f8, p, g, copy):
    rng = np.random.Generator(np.random.Philox(17))
    tensors = [Tensor(rng, n, p, g, f8, copy, lr_scale=1.0 + 0.25 * (i % 3), decay=0.1 * (i % 2)) for i, n in enumerate(SIZES)]
    run(tensors, "%s %s %s" % (p, g, "f8" if f8 else "f32"), steps=3, grad_scale=0.25)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_alignments(f8, off):
    rng = np.random.Generator(np.random.Philox(off))
    run([Tensor(rng, n, g="f16", f8=f8, copy=True, off=off) for n in (1, 7, 256, 1000, 5003)], "off by %d" % off)


@pytest.mark.parametrize("count", [1, 2, 63, 64, 65, 128, 129, 300, 4097, 5000])
def test_many_tensors_empty_ones_among_them(count):
    """Lists around the sizes at which the search for a block's tensor takes another look."""
    rng = np.random.Generator(np.random.Philox(count))
    tensors = []
    for i in range(count):
        n = int(rng.integers(0, 4)) * (0 if i % 5 == 0 else 1) if count > 1000 else int(rng.choice([0, 1, 200, 1024, 1500]))
        tensors.append(Tensor(rng, n, f8=i % 2 == 1, decay=0.01))
    run(tensors, "%d tensors" % count)


@pytest.mark.parametrize("f8", [False, True])
def test_large_lists_take_more_rows_to_a_block(f8):
    rng = np.random.Generator(np.random.Philox(3))
    run([Tensor(rng, n, g="f16", f8=f8, copy=True, decay=0.01) for n in (1, 2500001, 4097, 700, 300000, 16)], "large", steps=2)


def test_mixed_kinds_in_one_list():
    rng = np.random.Generator(np.random.Philox(4))
    tensors = [Tensor(rng, 1 + 371 * i, "f16" if i % 3 == 0 else "f32", "f16" if i % 2 else "f32", f8=i % 4 < 2, copy=i % 3 == 1)
               for i in range(24)]
    run(tensors, "mixed", steps=2)


@pytest.mark.parametrize("f8", [False, True])
def test_gradients_that_are_not_finite(f8):
    rng = np.random.Generator(np.random.Philox(5))
    tensors = [Tensor(rng, 3000, f8=f8, decay=0.1), Tensor(rng, 10, f8=f8)]
    g = tensors[0].g.t
    g[7], g[300], g[301], g[2999] = float("nan"), float("inf"), -float("inf"), 3e20
    g[1500] = 1e21                    # 0.001 of its square overflows; that of 3e20, at the other end, does not
    before = [t.p.host().copy() for t in tensors]
    run(tensors, "not finite", steps=2)
    for i in (7, 300, 301, 1500):
        assert tensors[0].p.host()[i] == before[0][i]
    before = [t.p.host().copy() for t in tensors]
    run(tensors, "scale not finite", grad_scale=float("inf"))
    assert all(np.array_equal(t.p.host(), b) for t, b in zip(tensors, before))


@pytest.mark.parametrize("spread", [1e-18, 1e-12, 1e-4, 1e6, 1e17])
@pytest.mark.parametrize("f8", [False, True])
def test_magnitudes(spread, f8):
    """Moments down to the subnormals and up to the largest."""
    rng = np.random.Generator(np.random.Philox(6))
    run([Tensor(rng, 2000, f8=f8, spread=spread), Tensor(rng, 500, f8=f8, spread=spread, fresh=True)], "spread %g" % spread, steps=3)


@pytest.mark.parametrize("spread", [1e-12, 1e-3, 1.0, 1e9])
def test_codes_follow_from_the_rounded_root(spread):
    """Bit by bit over many elements and steps: a root that is one unit off changes one code in a hundred thousand."""
    rng = np.random.Generator(np.random.Philox(12))
    t = Tensor(rng, 1 << 20, g="f16" if spread == 1.0 else "f32", f8=True, spread=spread)
    plan, ws = make_plan([t])
    h = dict(HYPER)
    hy = fq.FqAdamW(**h)
    for i in range(3):
        h["step"] = hy.step = 50 + i
        want = t.reference(h, 0, None)
        fq.fq_adamw_step(plan, hy)
        torch.cuda.synchronize()
        t.compare(want, "rounded root, step %d" % i)
        assert np.array_equal(t.v.host(), want["v8"].astype(np.float32))
    fq.fq_adamw_destroy(plan)


@pytest.mark.parametrize("f8", [False, True])
def test_fresh_states_zero_gradients_and_other_constants(f8):
    rng = np.random.Generator(np.random.Philox(7))
    tensors = [Tensor(rng, 1500, f8=f8, fresh=True), Tensor(rng, 900, f8=f8, spread=0.0), Tensor(rng, 900, f8=f8, spread=0.0, decay=0.3)]
    tensors[0].g.t[::3] = 0.0
    run(tensors, "fresh", steps=4, step=1)
    run(tensors, "no momentum", beta1=0.0, beta2=0.0, eps=1e-3)
    run(tensors, "negative rate", lr=-1e-2, beta2=0.99)


def test_stochastic_rounding_is_unbiased_and_the_averages_move():
    """One value for all elements: the mean of the codes is the value, to five standard deviations of a mean of n code
    steps; and after many steps with a constant square of the gradient v has come near it, although every single step is
    smaller than half a code step."""
    n = 1 << 18
    rng = np.random.Generator(np.random.Philox(8))
    t = Tensor(rng, n, f8=True, fresh=True)
    t.g.t.fill_(0.37)
    plan, ws = make_plan([t])
    h = fq.FqAdamW(lr=0.0, beta1=0.9, beta2=0.999, step=1, seed=5)
    fq.fq_adamw_step(plan, h)
    m = t.m.host().reshape(-1, 256) * t.ms.host()[:, None]
    r = t.v.host().reshape(-1, 256) * t.vs.host()[:, None]
    for got, want in ((m, np.float64(np.float32(0.1)) * 0.37), (r, np.sqrt(0.001) * 0.37)):
        step = 2.0 ** (np.floor(np.log2(want)) - 3)
        assert set(np.unique(np.round(got / step - np.floor(want / step)))) <= {0.0, 1.0}
        assert abs(got.mean(dtype=np.float64) - want) <= 5 * 0.5 * step / np.sqrt(n) + 2.0 ** -16 * step + 1e-6 * want
    for i in range(2, 4000):
        h.step = i
        fq.fq_adamw_step(plan, h)
    torch.cuda.synchronize()
    r = t.v.host().reshape(-1, 256) * t.vs.host()[:, None]
    # 1 - 0.999^4000 = 0.98; rounding adds its variance to v, at most (1/8)^2/4 of it per changed code
    assert 0.93 * 0.37 <= r.mean() <= 1.10 * 0.37
    m = t.m.host().reshape(-1, 256) * t.ms.host()[:, None]
    assert abs(m.mean() - 0.37) <= 0.01 * 0.37
    fq.fq_adamw_destroy(plan)


@pytest.mark.parametrize("f8", [False, True])
def test_the_same_bits_every_time_on_streams_and_in_graphs(f8):
    rng = np.random.Generator(np.random.Philox(9))
    tensors = [Tensor(rng, n, g="f16", f8=f8, copy=True, decay=0.01) for n in (5000, 3, 70000)]
    state = [x.bytes for t in tensors for x in t.all()]
    saved = [b.clone() for b in state]

    def restore():
        for b, s in zip(state, saved):
            b.copy_(s)

    plan, ws = make_plan(tensors)
    h = fq.FqAdamW(**HYPER)
    fq.fq_adamw_step(plan, h)
    torch.cuda.synchronize()
    first = [b.clone() for b in state]
    restore()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fq.fq_adamw_step(plan, h)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(state, first))
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.fq_adamw_step(plan, h)
    for turn in range(5):
        restore()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(state, first)), "replay %d" % turn
    restore()
    h.seed += 1                       # other random numbers: other codes, the same parameters
    fq.fq_adamw_step(plan, h)
    torch.cuda.synchronize()
    assert torch.equal(tensors[0].p.bytes, first[0])
    assert f8 != torch.equal(tensors[2].m.bytes, first[[id(x) for t in tensors for x in t.all()].index(id(tensors[2].m))])
    fq.fq_adamw_destroy(plan)

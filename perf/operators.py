"""The work of the int8 linear layer and of the multi-tensor AdamW step: their cases, their plain forms and their
values in 64 bits.

Every case is a dict of plain values.  `op` says which operator one pass calls:

  linear   y = xs * ws * (codes of x) (codes of w)^T + bias by fq_linear_forward: m tokens of k values against n
           channels.  `x` is the tokens' type: float16 / float32 are quantized row by row within the call, int8 are
           codes that come with their scales (`scales`: one per token, or one for all).
  adamw    one AdamW step over a list of tensors by fq_adamw_step, with the moments in FP32 or in FP8 (e4m3 codes, a
           power-of-two scale per 256 elements, stochastic rounding from a counter-based hash).  `sizes` is
           "front_end" (weights, biases and both kinds of scale parameters of the 22 convolutions of the front end,
           channels times `width`) or "mixed" (`tensors` tensors of `elements` elements together).

Where `own` is false, run() computes the plain form: elementary torch operations in 32 bits.  Both forms work on the
same state.  All random numbers (inputs and the seed of the stochastic rounding) come from the seed of prepare().
"""
import math
import random

import torch

own = False

# The 22 convolutions of the front end: two encoders of 11 that differ in their last output width
# (channels in, channels out, kernel).
_ENCODER = [(3, 32, 7)] + [(32, 32, 3)] * 4 + [(32, 64, 3), (32, 64, 1)] + [(64, 64, 3)] * 3
_FRONT_END = _ENCODER + [(64, 128, 1)] + _ENCODER + [(64, 384, 1)]

_BLOCK = 256                 # elements that share a scale of an 8-bit state
_HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
_DECAY = 0.01
_GRAD_SCALE = 1.0 / 1024.0   # the gradients come with a loss scale
_FIRST_STEP = 101            # the moments below are those of a run that has lasted a while
_FLT_MIN = 1.1754943508222875e-38


def listed():
    return [
        # decoding one token: the weights' bytes, and latency
        dict(name="linear_one_token", op="linear", m=1, k=4096, n=4096, x="float16", y="float16", bias=False,
             scales="token"),
        # decoding a batch of twenty streams through a widening layer
        dict(name="linear_few_tokens", op="linear", m=20, k=4096, n=16384, x="float16", y="float16", bias=False,
             scales="token"),
        # a prompt of a few hundred tokens
        dict(name="linear_prompt", op="linear", m=600, k=4096, n=4096, x="float16", y="float16", bias=True,
             scales="token"),
        # 1x1 convolution of the 384-channel feature map: 120 x 160 positions
        dict(name="linear_feature_map", op="linear", m=19200, k=384, n=384, x="float16", y="float16", bias=True,
             scales="token"),
        # 3x3 convolution of 384 channels over unfolded patches: codes and one learned scale, as fq_forward gives them
        dict(name="linear_conv_codes", op="linear", m=19200, k=3456, n=384, x="int8", y="float16", bias=True,
             scales="tensor"),
        # nothing is a whole number of tiles or vectors, FP32 in and out
        dict(name="linear_ragged", op="linear", m=1201, k=1155, n=257, x="float32", y="float32", bias=True,
             scales="token"),
        # a long batch through a square layer: the matrix cores
        dict(name="linear_large", op="linear", m=8192, k=8192, n=8192, x="float16", y="float16", bias=False,
             scales="token"),
        # training the front end: 88 tensors, most of them tiny; launches and latency
        dict(name="adamw_front_end", op="adamw", sizes="front_end", width=1, params="float32", grads="float32",
             states="float32", copy=False),
        # the same four times as wide, FP16 gradients, 8-bit moments and an FP16 copy of the weights
        dict(name="adamw_front_end_f8", op="adamw", sizes="front_end", width=4, params="float32", grads="float16",
             states="float8", copy=True),
        # a fine-tuning run that keeps nothing but FP16 weights and 8-bit moments
        dict(name="adamw_fp16_f8", op="adamw", sizes="mixed", tensors=48, elements=20000000, mix=3, params="float16",
             grads="float16", states="float8", copy=False),
        # a large model's shard, classical and with 8-bit moments
        dict(name="adamw_large_f32", op="adamw", sizes="mixed", tensors=64, elements=120000000, mix=1,
             params="float32", grads="float32", states="float32", copy=False),
        dict(name="adamw_large_f8", op="adamw", sizes="mixed", tensors=64, elements=240000000, mix=2,
             params="float32", grads="float16", states="float8", copy=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A size: odd ones and whole numbers of 16, 64 and 128 among them."""
    v, grain = _log(rng, lo, hi), rng.choice([1, 1, 16, 64, 128])
    v = max(lo, v // grain * grain)
    return v + 1 if v == 3072 else v


def draw(rng):
    if rng.random() < 0.6:
        x = rng.choice(["float16", "float16", "float32", "int8"])
        m, k, n = _extent(rng, 1, 20000), _extent(rng, 16, 8192), _extent(rng, 16, 16384)
        while 2.0 * m * n * k > 1.0e12:
            m, n = (m + 1) // 2, (n + 1) // 2
        return dict(op="linear", m=m, k=k, n=n, x=x, y=rng.choice(["float16", "float16", "float32"]),
                    bias=rng.random() < 0.5, scales=rng.choice(["token", "tensor"]) if x == "int8" else "token")
    params, states = rng.choice(["float32", "float32", "float16"]), rng.choice(["float32", "float8", "float8"])
    grads = "float16" if params == "float16" else rng.choice(["float32", "float16"])
    copy = params == "float32" and rng.random() < 0.5
    if rng.random() < 0.25:
        return dict(op="adamw", sizes="front_end", width=rng.randint(1, 9), params=params, grads=grads, states=states,
                    copy=copy)
    return dict(op="adamw", sizes="mixed", tensors=_log(rng, 1, 300), elements=_log(rng, 20000, 100000000),
                mix=rng.randint(10, 1 << 20), params=params, grads=grads, states=states, copy=copy)


def _type(name):
    return {"float16": torch.float16, "float32": torch.float32, "int8": torch.int8}[name]


def _bytes(name):
    return {"float8": 1, "int8": 1, "float16": 2, "float32": 4}[name]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


# --------------------------------------------------------------------------------------------------------- inputs
def _linear_inputs(case, seed):
    """Tokens with a magnitude each and a few channels ten times as large, weights of variance 2 / k as codes with the
    scale of each channel's largest magnitude."""
    gen = _generator(seed)
    m, n, k = case["m"], case["n"], case["k"]
    given = {"bias": _randn(gen, n) if case["bias"] else None}
    w = _randn(gen, n, k) * math.sqrt(2.0 / k)
    scale = w.abs().amax(1) / 127.0
    given["w"] = torch.round(w / scale[:, None]).clamp_(-127, 127).to(torch.int8)
    given["w_scale"] = scale
    del w
    x = _randn(gen, m, k)
    x *= torch.exp(0.5 * _randn(gen, m, 1))
    x *= torch.where(torch.rand((1, k), generator=gen, device="cuda") < 0.01, 10.0, 1.0)
    given["x_scale"] = None
    if case["x"] == "int8":
        scale = x.abs().amax(1) / 127.0 if case["scales"] == "token" else x.abs().amax().reshape(1) / 127.0
        x = torch.round(x / scale[:, None]).clamp_(-127, 127)
        given["x_scale"] = scale
    given["x"] = x.to(_type(case["x"]))
    return given


def _sizes(case):
    """The list's tensors: (elements, weight decay)."""
    got = []
    if case["sizes"] == "front_end":
        wide = case["width"]
        for ci, co, kernel in _FRONT_END:
            ci, co = ci if ci == 3 else ci * wide, co * wide
            got += [(ci * co * kernel * kernel, _DECAY), (co, 0.0), (co, 0.0), (1, 0.0)]   # weight, bias, thetas
    else:
        rng = random.Random(case["mix"])
        share = [math.exp(rng.uniform(0.0, 6.0)) for _ in range(case["tensors"])]
        for s in share:
            size = max(1, int(case["elements"] * s / sum(share)))
            got.append((size if size != 3072 else 3073, _DECAY if rng.random() < 0.7 else 0.0))
    return got


def _places(case):
    """(first block, elements, weight decay) of each tensor in the flat buffers, where every tensor begins a block, and
    the number of blocks."""
    places, at = [], 0
    for size, decay in _sizes(case):
        places.append((at, size, decay))
        at += -(-size // _BLOCK)
    return places, at


def _adamw_inputs(case, seed):
    """Flat buffers, zero behind every tensor's last element: parameters, gradients whose magnitude differs from block
    to block, and moments that belong to such gradients (in FP8: codes and scales of them)."""
    gen = _generator(seed)
    places, blocks = _places(case)
    total = blocks * _BLOCK
    size = torch.tensor([p[1] for p in places], device="cuda")
    count = (size + _BLOCK - 1) // _BLOCK
    first = torch.repeat_interleave(torch.cumsum(count, 0) - count, count)
    left = torch.repeat_interleave(size, count) - (torch.arange(blocks, device="cuda") - first) * _BLOCK
    there = torch.arange(_BLOCK, device="cuda")[None, :] < left[:, None]
    spread = torch.exp(1.5 * _randn(gen, blocks, 1))
    noise = lambda s: torch.where(there, _randn(gen, blocks, _BLOCK) * s, 0.0)   # noqa: E731
    given = {"p": noise(0.05).reshape(total).to(_type(case["params"])),
             "g": noise(spread).reshape(total).to(_type(case["grads"])), "seed": int(seed)}
    m = noise(0.2 * _GRAD_SCALE * spread)
    v = (m * 3.0 + noise(_GRAD_SCALE * spread)).square()
    given["decay"] = torch.repeat_interleave(torch.tensor([p[2] for p in places], device="cuda"), count)
    given["grad_scale"] = torch.full((1,), _GRAD_SCALE, device="cuda")
    if case["states"] == "float8":
        for name, value in (("m", m), ("v", v.sqrt())):
            scale = torch.exp2(torch.ceil(torch.log2(value.abs().amax(1).clamp_min(1e-30) / 448.0)))
            given[name] = (value / scale[:, None]).reshape(total).to(torch.float8_e4m3fn)
            given[name + "_scale"] = scale
    else:
        given["m"], given["v"] = m.reshape(total), v.reshape(total)
    given["copy"] = given["p"].half() if case["copy"] else None
    return given


def prepare(case, seed):
    if case["op"] == "linear":
        state = _linear_inputs(case, seed)
        state["y"] = torch.zeros((case["m"], case["n"]), dtype=_type(case["y"]), device="cuda")
        if own:
            from paper_2511_12653_amd import binding as fq
            state["d"] = fq.FqLinear.from_torch(state["x"], state["w"], state["w_scale"], state["y"],
                                                bias=state["bias"], x_scale=state["x_scale"])
            state["workspace"] = torch.empty(fq.fq_linear_workspace_bytes(state["d"]), dtype=torch.uint8, device="cuda")
    else:
        state = _adamw_inputs(case, seed)
        state["step"] = _FIRST_STEP - 1
        if own:
            from paper_2511_12653_amd import binding as fq
            params = []
            for at, size, decay in _places(case)[0]:
                part = lambda name: state[name][at * _BLOCK:at * _BLOCK + size]     # noqa: E731
                scales = {}
                if case["states"] == "float8":
                    scales = {s: state[s][at:at - (-size // _BLOCK)] for s in ("m_scale", "v_scale")}
                params.append(fq.FqParam.from_torch(part("p"), part("g"), part("m"), part("v"), weight_decay=decay,
                                                    p16=part("copy") if case["copy"] else None, **scales))
            workspace = torch.empty(fq.fq_adamw_workspace_bytes(params), dtype=torch.uint8, device="cuda")
            state["plan"] = fq.fq_adamw_create(params, workspace)
            state["hyper"] = fq.FqAdamW(step=0, seed=state["seed"], grad_scale=state["grad_scale"], **_HYPER)
            state["workspace"] = workspace
    state["case"] = case
    return state


# ---------------------------------------------------------------------------------------------------------- passes
def run(state):
    case = state["case"]
    if case["op"] == "linear":
        if own:
            from paper_2511_12653_amd import binding as fq
            fq.fq_linear_forward(state["d"], state["workspace"])
            return state["y"]
        return _plain_linear(state, _type(case["y"]))
    state["step"] += 1
    if own:
        from paper_2511_12653_amd import binding as fq
        state["hyper"].step = state["step"]
        fq.fq_adamw_step(state["plan"], state["hyper"])
    else:
        _plain_adamw(state)
    return {name: state[name] for name in ("p", "m", "v", "m_scale", "v_scale", "copy") if state.get(name) is not None}


def _plain_linear(state, y_type):
    x = state["x"].float()
    scale = state["x_scale"]
    if scale is None:
        largest = x.abs().amax(1)
        scale = largest / torch.full_like(largest, 127.0)
        scale = torch.where(largest < 127.0 * _FLT_MIN, torch.zeros_like(scale), scale)
        x = torch.round(x / scale[:, None]).clamp_(-127.0, 127.0)
        x = torch.where(scale[:, None] == 0.0, torch.zeros_like(x), x)
    y = torch.matmul(x, state["w"].float().t())
    y *= scale[:, None] * state["w_scale"][None, :]
    if state["bias"] is not None:
        y += state["bias"][None, :]
    return y.to(y_type)


def _float32(x):
    """x rounded to a binary32 value."""
    return torch.tensor(x, dtype=torch.float64).float().item()


def _key(seed, step):
    """The key of a step's random numbers: 64-bit products of seed and step, mixed down to 32 bits."""
    k = (seed * 0x9E3779B97F4A7C15 + step * 0xD1B54A32D192ED03) % (1 << 64)
    k = ((k ^ (k >> 32)) * 0x9E3779B97F4A7C15) % (1 << 64)
    return k >> 32


def _signed(x):
    return x - (1 << 32) if x >= 1 << 31 else x


def _random_bits(count, key):
    """32 random bits for each of `count` places: the place's hash under the key, in wrapping 32-bit products."""
    x = torch.arange(count, dtype=torch.int32, device="cuda") * _signed(0x9E3779B1) + _signed(key)
    x = (x ^ ((x >> 16) & 0xFFFF)) * 0x6A09E667
    x = (x ^ ((x >> 15) & 0x1FFFF)) * _signed(0xBB67AE85)
    return x ^ ((x >> 16) & 0xFFFF)


def _power(largest, most):
    """e of the least power of two with largest <= most * 2^e, at least -126."""
    mantissa, exponent = torch.frexp(largest)
    limit, shift = math.frexp(most)
    e = exponent - shift + (mantissa > limit).to(exponent.dtype)
    return torch.where(largest > 0, e, -126).clamp_(-126, 126)


def _encode(value, e, bits):
    """value / 2^e as e4m3 by stochastic rounding: `bits` (16 of them) is added below the third mantissa bit."""
    a = value.abs() * torch.exp2(-e.float())[:, None]
    low = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0)         # there the steps are those of the binade above
    z = ((a + low).view(torch.int32) + (bits * 16 + 8)) & ~0xFFFFF
    return torch.copysign(z.view(torch.float32) - low, value)


def _plain_adamw(state):
    h, t = _HYPER, state["step"]
    f8 = "m_scale" in state
    blocks = state["decay"].numel()
    wide = lambda name: state[name].float().reshape(blocks, _BLOCK)     # noqa: E731
    p, m, v, g = wide("p"), wide("m"), wide("v"), wide("g") * state["grad_scale"]
    if f8:
        m = m * state["m_scale"][:, None]
        v = (v * state["v_scale"][:, None]).square()
    m1 = m * _float32(h["beta1"]) + g * _float32(1.0 - h["beta1"])
    v1 = v * _float32(h["beta2"]) + g * _float32(1.0 - h["beta2"]) * g
    fine = torch.isfinite(v1)
    m1, v1 = torch.where(fine, m1, m), torch.where(fine, v1, v)
    root = v1.sqrt()
    below = root * _float32(1.0 / math.sqrt(1.0 - h["beta2"] ** t)) + _float32(h["eps"])
    keep = 1.0 - _float32(h["lr"]) * state["decay"][:, None]
    p1 = p * keep - (m1 / below) * _float32(h["lr"] / (1.0 - h["beta1"] ** t))
    p1 = torch.where(fine, p1, p)
    if f8:
        bits = _random_bits(blocks * _BLOCK, _key(state["seed"], t)).reshape(blocks, _BLOCK)
        e = _power(m1.abs().amax(1), 448.0)
        m1 = _encode(m1, e, bits & 0xFFFF)
        state["m_scale"].copy_(torch.exp2(e.float()))
        # the greatest root is at most 448 * 2^e where the greatest v is at most (448 * 2^e)^2
        e = torch.div(_power(v1.amax(1), 448.0 ** 2) + 1, 2, rounding_mode="floor")
        code = _encode(root, e, (bits >> 16) & 0xFFFF)
        v1 = torch.where((v1 > 0) & (code == 0), 2.0 ** -9, code)
        state["v_scale"].copy_(torch.exp2(e.float()))
    state["p"].copy_(p1.reshape(-1))
    state["m"].copy_(m1.reshape(-1))
    state["v"].copy_(v1.reshape(-1))
    if state["copy"] is not None:
        state["copy"].copy_(p1.reshape(-1))


# ----------------------------------------------------------------------------------------- what a pass has to do
def work(case):
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        scales = n + (n if case["bias"] else 0) + (0 if case["x"] != "int8" else m if case["scales"] == "token" else 1)
        return dict(bytes=float(m * k * _bytes(case["x"]) + n * k + m * n * _bytes(case["y"]) + 4 * scales),
                    flops=2.0 * m * n * k)
    each = 2 * _bytes(case["params"]) + _bytes(case["grads"]) + 4 * _bytes(case["states"]) + (2 if case["copy"] else 0)
    sizes = [s for s, _ in _sizes(case)]
    scales = sum(-(-s // _BLOCK) for s in sizes) * 16 if case["states"] == "float8" else 0
    return dict(bytes=float(sum(sizes) * each + scales), flops=20.0 * sum(sizes))


# ------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    return _exact_linear(case, seed) if case["op"] == "linear" else _exact_adamw(case, seed)


def _exact_linear(case, seed):
    given = _linear_inputs(case, seed)
    x, w = given["x"].double(), given["w"].double()
    y = torch.empty((case["m"], case["n"]), dtype=torch.float64, device="cuda")
    for rows in torch.arange(case["m"], device="cuda").split(4096):
        part = x[rows]
        if given["x_scale"] is None:
            top = part.abs().max(dim=1, keepdim=True).values
            scale = top / 127.0
            part = torch.where(top > 0, torch.round(part / scale), torch.zeros_like(part))
        else:
            scale = given["x_scale"].double().reshape(-1, 1)
            scale = scale[rows] if scale.numel() > 1 else scale
        y[rows] = (part @ w.t()) * scale * given["w_scale"].double()
    return y if given["bias"] is None else y + given["bias"].double()


def _exact_rounding(value, bits, least):
    """(values of the e4m3 codes, scales): stochastic rounding down of a + u steps, u = (bits + 1/2) / 2^16.  Scales
    begin at 2^least."""
    top = value.abs().amax(1)
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448.0)).clamp_(min=least)
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1.0, e)
    a = value.abs() / torch.exp2(e)[:, None]
    step = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3.0)
    code = torch.floor(a / step + (bits.double() + 0.5) / 65536.0) * step
    return code * torch.sign(value), torch.exp2(e)


def _exact_adamw(case, seed):
    given = _adamw_inputs(case, seed)
    h, t, f8 = _HYPER, _FIRST_STEP, case["states"] == "float8"
    blocks = given["decay"].numel()
    out = {"p": torch.empty(blocks * _BLOCK, dtype=torch.float64, device="cuda")}
    for name in ("m", "v") + (("copy",) if case["copy"] else ()):
        out[name] = torch.empty_like(out["p"])
    for name in ("m_scale", "v_scale") if f8 else ():
        out[name] = torch.empty(blocks, dtype=torch.float64, device="cuda")
    random_bits = _random_bits(blocks * _BLOCK, _key(given["seed"], t)) if f8 else None
    for at in range(0, blocks, 1 << 16):
        some = slice(at, min(blocks, at + (1 << 16)))
        flat = slice(some.start * _BLOCK, some.stop * _BLOCK)
        part = lambda name: given[name][flat].double().reshape(-1, _BLOCK)     # noqa: E731
        p, m, v, g = part("p"), part("m"), part("v"), part("g") * _GRAD_SCALE
        if f8:
            m, v = m * given["m_scale"][some, None].double(), (v * given["v_scale"][some, None].double()) ** 2
        m = h["beta1"] * m + (1.0 - h["beta1"]) * g
        v = h["beta2"] * v + (1.0 - h["beta2"]) * g * g
        fraction = (m / (1.0 - h["beta1"] ** t)) / ((v / (1.0 - h["beta2"] ** t)).sqrt() + h["eps"])
        p = p - h["lr"] * given["decay"][some, None].double() * p - h["lr"] * fraction
        if f8:
            bits = random_bits[flat].reshape(-1, _BLOCK).long()
            m, out["m_scale"][some] = _exact_rounding(m, bits & 0xFFFF, -126.0)
            code, out["v_scale"][some] = _exact_rounding(v.sqrt(), (bits >> 16) & 0xFFFF, -63.0)
            v = torch.where((v > 0) & (code == 0), 2.0 ** -9, code)
        for name, value in (("p", p), ("m", m), ("v", v), ("copy", p)):
            if name in out:
                out[name][flat] = value.reshape(-1)
    return out

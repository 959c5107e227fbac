"""The work of layer norm, of dropout and of low-rank adapters beside the int8 linear layer: their cases, their plain
forms and their values in 64 bits.

Every case is a dict of plain values.  `op` says which operator one pass calls:

  norm           y = (x - mean) * rstd * weight + bias by fq_norm_forward: rows of `width` values.  `y` is float16 /
                 float32, or int8: codes with a scale per row, what the int8 linear layer takes.
  norm_backward  the gradients of x, weight and bias by fq_norm_backward.
  dropout        y = x / (1 - p) where a counter-based generator says so, else 0, plus a residual, by fq_dropout.  With
                 no residual this is the backward pass, too: the same call on the gradient.
  adapters       y = base + scale * (x a^T) b^T by fq_adapters_forward: `m` tokens of `k` values, `n` channels, every
                 token with one of `count` adapters of rank `rank`, or none.  `order` says how tokens come: "runs" (the
                 tokens of a request one after the other, each request with its adapter) or "mixed" (decoding: one token
                 of every request).

Where `own` is false, run() computes the plain form: elementary torch operations in 32 bits (codes: in 64, since values
next to the border of two codes decide).  All random numbers (inputs and the seed of the generator) come from the seed of
prepare().
"""
import math

import torch

own = False

_EPS = 1e-5
_FLT_MIN = 1.1754943508222875e-38
_STEP = 100                  # of the generator: the hundredth step of a run
_CHUNK = 1 << 22             # elements at a time in 64 bits


def listed():
    return [
        # one token of a decoding loop on its way into an int8 layer: latency
        dict(name="norm_token_codes", op="norm", rows=1, width=4096, x="float16", y="int8", w="float32"),
        # the same for a prompt of a few hundred tokens, out of a residual stream in FP32
        dict(name="norm_prompt_codes", op="norm", rows=600, width=4096, x="float32", y="int8", w="float32"),
        # training's forward pass over a long batch
        dict(name="norm_large", op="norm", rows=32768, width=8192, x="float16", y="float16", w="float32"),
        # training on the 384-channel feature map: 120 x 160 positions
        dict(name="norm_backward_feature_map", op="norm_backward", rows=19200, width=384, x="float16", y="float16",
             w="float32"),
        # nothing is a whole number of vectors, FP32
        dict(name="norm_backward_ragged", op="norm_backward", rows=1201, width=1155, x="float32", y="float32",
             w="float32"),
        # training's backward pass over a long batch of wide rows
        dict(name="norm_backward_large", op="norm_backward", rows=16384, width=4096, x="float16", y="float16",
             w="float32"),
        # a small layer's activations: the launch
        dict(name="dropout_small", op="dropout", n=24611, x="float32", y="float32", p=0.1, residual=False),
        # the training batch of 15 x 128 x 120 x 160, added to the residual stream
        dict(name="dropout_batch", op="dropout", n=36864000, x="float16", y="float16", p=0.1, residual=True),
        # decoding one token with its user's adapter
        dict(name="adapters_token", op="adapters", m=1, k=4096, n=4096, count=8, rank=16, x="float16", y="float16",
             base="float16", order="mixed"),
        # decoding 48 streams, each with one of 32 adapters or none
        dict(name="adapters_batch", op="adapters", m=48, k=4096, n=4096, count=32, rank=16, x="float16", y="float16",
             base="float16", order="mixed"),
        # prompts of a few requests behind a norm that gives codes; ragged
        dict(name="adapters_prompt", op="adapters", m=601, k=4096, n=4096, count=6, rank=24, x="int8", y="float16",
             base="float32", order="runs"),
        # long prompts through wide layers
        dict(name="adapters_large", op="adapters", m=8192, k=8192, n=8192, count=8, rank=64, x="float16", y="float16",
             base="float16", order="runs"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A size: odd ones and whole numbers of 8, 64 and 128 among them."""
    v, grain = _log(rng, lo, hi), rng.choice([1, 1, 8, 64, 128])
    return max(lo, v // grain * grain)


def draw(rng):
    kind = rng.random()
    if kind < 0.45:
        rows, width = _log(rng, 1, 65536), _extent(rng, 16, 16384)
        while rows * width > 67000000:
            rows = (rows + 1) // 2
        x = rng.choice(["float16", "float16", "float32"])
        w = rng.choice(["float32", "float32", "float16"])
        if rng.random() < 0.5:
            return dict(op="norm", rows=rows, width=width, x=x, y=rng.choice(["float16", "float32", "int8", "int8"]),
                        w=w)
        return dict(op="norm_backward", rows=rows, width=width, x=x, y=rng.choice([x, x, "float16", "float32"]), w=w)
    if kind < 0.65:
        x = rng.choice(["float16", "float16", "float32"])
        return dict(op="dropout", n=_log(rng, 1000, 60000000), x=x, y=rng.choice([x, x, "float16", "float32"]),
                    p=rng.choice([0.05, 0.1, 0.1, 0.2, 0.5]), residual=rng.random() < 0.5)
    m, k, n = _log(rng, 1, 8192), _extent(rng, 64, 8192), _extent(rng, 64, 8192)
    rank, count = rng.choice([4, 8, 8, 16, 16, 32, 64, 128, rng.randint(1, 64)]), _log(rng, 1, 64)
    while count * rank > 1024:
        count = (count + 1) // 2
    while float(m) * (k + n) * count * rank > 4.0e10:
        m, count = (m + 1) // 2, (count + 1) // 2
    return dict(op="adapters", m=m, k=k, n=n, count=count, rank=rank,
                x=rng.choice(["float16", "float16", "int8", "float32"]), y=rng.choice(["float16", "float16", "float32"]),
                base=rng.choice(["float16", "float32"]), order=rng.choice(["runs", "mixed"]))


def _type(name):
    return {"float16": torch.float16, "float32": torch.float32, "int8": torch.int8}[name]


def _bytes(name):
    return {"int8": 1, "float16": 2, "float32": 4}[name]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rand(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


# --------------------------------------------------------------------------------------------------------- inputs
def _tokens(gen, rows, width):
    """Rows with a magnitude and a mean each and a few channels ten times as large."""
    x = _randn(gen, rows, width)
    x *= torch.where(_rand(gen, 1, width) < 0.01, 10.0, 1.0)
    x *= torch.exp(0.5 * _randn(gen, rows, 1))
    x += 0.3 * _randn(gen, rows, 1)
    return x


def _norm_inputs(case, seed):
    """Tokens, a weight near one, a bias near zero; for the backward pass gradients with a magnitude per row and the
    forward pass's statistics (mean and 1 / deviation)."""
    gen = _generator(seed)
    rows, width = case["rows"], case["width"]
    given = {"x": _tokens(gen, rows, width).to(_type(case["x"])),
             "weight": (1.0 + 0.2 * _randn(gen, width)).to(_type(case["w"])),
             "bias": (0.1 * _randn(gen, width)).to(_type(case["w"]))}
    if case["op"] == "norm_backward":
        gy = _randn(gen, rows, width)
        gy *= 0.1 * torch.exp(0.5 * _randn(gen, rows, 1))
        given["gy"] = gy.to(_type(case["y"]))
        del gy
        x = given["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = 1.0 / ((x - mean).square().mean(1, keepdim=True) + _EPS).sqrt()
        given["stats"] = torch.cat((mean, rstd), 1).contiguous()
    return given


def _dropout_inputs(case, seed):
    gen = _generator(seed)
    return {"x": _randn(gen, case["n"]).to(_type(case["x"])),
            "residual": _randn(gen, case["n"]).to(_type(case["y"])) if case["residual"] else None, "seed": int(seed)}


def _adapter_inputs(case, seed):
    """Tokens (codes: quantized row by row), what the shared projection gave for them, adapters whose products have the
    projection's magnitude, and each token's adapter (-1: none)."""
    gen = _generator(seed)
    m, k, n, count, rank = case["m"], case["k"], case["n"], case["count"], case["rank"]
    given = {"x_scale": None}
    x = _tokens(gen, m, k)
    if case["x"] == "int8":
        given["x_scale"] = x.abs().amax(1) / 127.0
        x = torch.round(x / given["x_scale"][:, None]).clamp_(-127, 127)
    given["x"] = x.to(_type(case["x"]))
    del x
    given["base"] = _randn(gen, m, n).to(_type(case["base"]))
    given["a"] = (_randn(gen, count, rank, k) / math.sqrt(k)).half()
    given["b"] = (_randn(gen, count, n, rank) / math.sqrt(rank)).half()
    given["scale"] = 0.5 + _rand(gen, count)
    if case["order"] == "runs":          # requests of random lengths, one adapter each
        requests = max(1, min(m, 2 * count))
        starts = torch.sort(torch.randint(0, m, (requests,), generator=gen, device="cuda")).values
        request = torch.searchsorted(starts, torch.arange(m, device="cuda"), right=True)
        of_request = torch.randint(-1, count, (requests + 1,), generator=gen, device="cuda")
        of_request[0] = count - 1
        given["ids"] = of_request[request].int()
    else:
        given["ids"] = torch.randint(-1 if m > 1 else 0, count, (m,), generator=gen, device="cuda").int()
    return given


def prepare(case, seed):
    if case["op"] in ("norm", "norm_backward"):
        state = _norm_inputs(case, seed)
        empty = lambda *shape, like: torch.zeros(shape, dtype=_type(like), device="cuda")     # noqa: E731
        rows, width = case["rows"], case["width"]
        if case["op"] == "norm":
            state["y"] = empty(rows, width, like=case["y"])
            if case["y"] == "int8":
                state["y_scale"] = torch.zeros(rows, device="cuda")
            else:
                state["stats"] = torch.zeros((rows, 2), device="cuda")
        else:
            state["gx"] = empty(rows, width, like=case["x"])
            state["gweight"], state["gbias"] = empty(width, like=case["w"]), empty(width, like=case["w"])
        if own:
            from paper_2511_12653_amd import binding as fq
            part = lambda *names: {name: state[name] for name in names if name in state}     # noqa: E731
            state["d"] = fq.FqNorm.from_torch(state["x"], eps=_EPS, **part("weight", "bias", "y", "y_scale", "stats", "gy",
                                                                           "gx", "gweight", "gbias"))
            if case["op"] == "norm_backward":
                state["workspace"] = torch.empty(fq.fq_norm_workspace_bytes(state["d"]), dtype=torch.uint8, device="cuda")
    elif case["op"] == "dropout":
        state = _dropout_inputs(case, seed)
        state["y"] = torch.zeros(case["n"], dtype=_type(case["y"]), device="cuda")
        if own:
            from paper_2511_12653_amd import binding as fq
            state["d"] = fq.FqDropout.from_torch(state["x"], state["y"], case["p"], state["seed"], step=_STEP,
                                                 residual=state["residual"])
    else:
        state = _adapter_inputs(case, seed)
        state["y"] = torch.zeros((case["m"], case["n"]), dtype=_type(case["y"]), device="cuda")
        if own:
            from paper_2511_12653_amd import binding as fq
            state["d"] = fq.FqAdapters.from_torch(state["x"], state["ids"], state["a"], state["b"], state["y"],
                                                  base=state["base"], scale=state["scale"], x_scale=state["x_scale"])
            state["workspace"] = torch.empty(fq.fq_adapters_workspace_bytes(state["d"]), dtype=torch.uint8, device="cuda")
    state["case"] = case
    return state


# ---------------------------------------------------------------------------------------------------------- passes
def run(state):
    case = state["case"]
    if case["op"] == "norm":
        if own:
            from paper_2511_12653_amd import binding as fq
            fq.fq_norm_forward(state["d"])
        elif case["y"] == "int8":
            state["y"], state["y_scale"] = _plain_norm_codes(state)
        else:
            state["y"], state["stats"] = _plain_norm(state, _type(case["y"]))
        return {name: state[name] for name in ("y", "y_scale", "stats") if name in state}
    if case["op"] == "norm_backward":
        if own:
            from paper_2511_12653_amd import binding as fq
            fq.fq_norm_backward(state["d"], state["workspace"])
            return {name: state[name] for name in ("gx", "gweight", "gbias")}
        return _plain_norm_backward(state)
    if case["op"] == "dropout":
        if own:
            from paper_2511_12653_amd import binding as fq
            fq.fq_dropout(state["d"])
            return state["y"]
        return _plain_dropout(state, case["p"], _type(case["y"]))
    if own:
        from paper_2511_12653_amd import binding as fq
        fq.fq_adapters_forward(state["d"], state["workspace"])
        return state["y"]
    return _plain_adapters(state, _type(case["y"]))


def _plain_norm(state, y_type):
    x = state["x"].float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = 1.0 / (x.square().mean(1, keepdim=True) + _EPS).sqrt()
    y = x * rstd * state["weight"].float() + state["bias"].float()
    return y.to(y_type), torch.cat((mean, rstd), 1)


def _plain_norm_codes(state):
    x = state["x"].double()
    x = x - x.mean(1, keepdim=True)
    rstd = 1.0 / (x.square().mean(1, keepdim=True) + _EPS).sqrt()
    y = (x * rstd * state["weight"].double() + state["bias"].double()).float()
    largest = y.abs().amax(1)
    scale = largest / torch.full_like(largest, 127.0)
    scale = torch.where(largest < 127.0 * _FLT_MIN, torch.zeros_like(scale), scale)
    codes = torch.round(y / scale[:, None]).clamp_(-127.0, 127.0)
    return torch.where(scale[:, None] == 0.0, torch.zeros_like(codes), codes).to(torch.int8), scale


def _plain_norm_backward(state):
    x, gy, mean, rstd = state["x"].float(), state["gy"].float(), state["stats"][:, :1], state["stats"][:, 1:]
    normed = (x - mean) * rstd
    a = gy * state["weight"].float()
    gx = rstd * (a - a.mean(1, keepdim=True) - normed * (a * normed).mean(1, keepdim=True))
    kind = state["weight"].dtype
    return {"gx": gx.to(state["x"].dtype), "gweight": (gy * normed).sum(0).to(kind), "gbias": gy.sum(0).to(kind)}


def _signed(x):
    return x - (1 << 32) if x >= 1 << 31 else x


def _keys(seed, step, high):
    """The two 32-bit keys of a step's random numbers (for places whose upper 32 bits are `high`)."""
    most = (1 << 64) - 1
    k = (seed * 0x9E3779B97F4A7C15 + step * 0xD1B54A32D192ED03 + high * 0x8CB92BA72F3D8DD7) & most
    k = ((k ^ (k >> 32)) * 0x9E3779B97F4A7C15) & most
    k = ((k ^ (k >> 29)) * 0xD1B54A32D192ED03) & most
    return k >> 32, (k ^ (k >> 32)) & 0xFFFFFFFF


def _random_bits(count, seed, step):
    """31 random bits for each of `count` places (under 2^32): the place's hash, in wrapping 32-bit products."""
    first, second = _keys(seed, step, 0)
    x = torch.arange(count, device="cuda").to(torch.int32) * _signed(0x9E3779B1) + _signed(first)
    x = (x ^ ((x >> 16) & 0xFFFF)) * 0x6A09E667
    x = ((x ^ ((x >> 15) & 0x1FFFF)) + _signed(second)) * _signed(0xBB67AE85)
    return (x >> 1) & 0x7FFFFFFF


def _plain_dropout(state, p, y_type):
    keep = _random_bits(state["x"].numel(), state["seed"], _STEP) >= round(p * (1 << 31))
    y = torch.where(keep, state["x"].float() * (1.0 / (1.0 - p)), 0.0)
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return y.to(y_type)


def _plain_adapters(state, y_type):
    """One product with all adapters, of which every token keeps its own."""
    a, b, ids = state["a"].float(), state["b"].float(), state["ids"]
    count, rank, k = a.shape
    x = state["x"].float()
    if state["x_scale"] is not None:
        x = x * state["x_scale"][:, None]
    t = torch.matmul(x, a.reshape(count * rank, k).t()).reshape(-1, count, rank)
    mine = ids[:, None] == torch.arange(count, device="cuda")[None, :]
    t = torch.where(mine[:, :, None], t * state["scale"][None, :, None], 0.0).reshape(-1, count * rank)
    y = torch.matmul(t, b.transpose(1, 2).reshape(count * rank, -1))
    return (state["base"].float() + y).to(y_type)


# ----------------------------------------------------------------------------------------- what a pass has to do
def work(case):
    if case["op"] in ("norm", "norm_backward"):
        each, rows, width = _bytes(case["x"]) + _bytes(case["y"]), case["rows"], case["width"]
        if case["op"] == "norm":
            return dict(bytes=float(rows * width * each + rows * (4 if case["y"] == "int8" else 8) +
                                    2 * width * _bytes(case["w"])), flops=8.0 * rows * width)
        return dict(bytes=float(rows * width * (each + _bytes(case["x"])) + 8 * rows + 3 * width * _bytes(case["w"])),
                    flops=14.0 * rows * width)
    if case["op"] == "dropout":
        each = _bytes(case["x"]) + _bytes(case["y"]) * (2 if case["residual"] else 1)
        return dict(bytes=float(case["n"] * each), flops=2.0 * case["n"])
    m, k, n = case["m"], case["k"], case["n"]
    used = min(m, case["count"])
    return dict(bytes=float(m * k * _bytes(case["x"]) + m * n * (_bytes(case["base"]) + _bytes(case["y"])) +
                            2 * used * case["rank"] * (k + n) + 4 * (m + used) + (4 * m if case["x"] == "int8" else 0)),
                flops=2.0 * m * case["rank"] * (k + n))


# ------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    return {"norm": _exact_norm, "norm_backward": _exact_norm_backward, "dropout": _exact_dropout,
            "adapters": _exact_adapters}[case["op"]](case, seed)


def _exact_norm(case, seed):
    given = _norm_inputs(case, seed)
    rows, width = case["rows"], case["width"]
    codes = case["y"] == "int8"
    stats = torch.empty((rows, 2), dtype=torch.float64, device="cuda")
    scale = torch.empty(rows, dtype=torch.float64, device="cuda")
    y = None if codes else torch.empty((rows, width), dtype=torch.float64, device="cuda")
    for at in torch.arange(rows, device="cuda").split(max(1, _CHUNK // width)):
        x = given["x"][at].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        stats[at, 0], stats[at, 1] = mean, (var + _EPS).rsqrt()
        part = torch.addcmul(given["bias"].double(), (x - mean[:, None]) * stats[at, 1:], given["weight"].double())
        scale[at] = part.abs().max(dim=1).values / 127.0
        if not codes:
            y[at] = part
    return {"y": None, "y_scale": scale} if codes else {"y": y, "stats": stats}


def _exact_norm_backward(case, seed):
    given = _norm_inputs(case, seed)
    rows, width = case["rows"], case["width"]
    gx = torch.empty((rows, width), dtype=torch.float64, device="cuda")
    gweight, gbias = torch.zeros((2, width), dtype=torch.float64, device="cuda")
    for at in torch.arange(rows, device="cuda").split(max(1, _CHUNK // width)):
        x, g = given["x"][at].double(), given["gy"][at].double()
        mean, rstd = given["stats"][at].double().unsqueeze(2).unbind(1)
        h = (x - mean) * rstd
        gweight += torch.einsum("ij,ij->j", g, h)
        gbias += g.sum(0)
        g *= given["weight"].double()
        inner = torch.linalg.vecdot(g, h).div(width).unsqueeze(1)
        gx[at] = (g - g.mean(1, keepdim=True) - inner * h) * rstd
    return {"gx": gx, "gweight": gweight, "gbias": gbias}


def _exact_dropout(case, seed):
    given = _dropout_inputs(case, seed)
    first, second = _keys(given["seed"], _STEP, 0)
    y = torch.empty(case["n"], dtype=torch.float64, device="cuda")
    low = 0xFFFFFFFF
    for at in torch.arange(case["n"], device="cuda").split(_CHUNK):
        h = (at * 0x9E3779B1 + first) & low          # in 64 bits: no product of two 32-bit numbers is cut off wrongly
        h = ((h ^ (h >> 16)) * 0x6A09E667) & low
        h = ((((h ^ (h >> 15)) + second) & low) * 0xBB67AE85) & low
        kept = (h.double() * 0.5).floor() >= round(case["p"] * 2.0 ** 31)
        part = kept.double() * given["x"][at].double() / (1.0 - case["p"])
        y[at] = part if given["residual"] is None else part + given["residual"][at].double()
    return y


def _exact_adapters(case, seed):
    given = _adapter_inputs(case, seed)
    y = given["base"].double()
    for adapter in range(case["count"]):
        rows = (given["ids"] == adapter).nonzero().flatten()
        x = given["x"][rows].double()
        if given["x_scale"] is not None:
            x = x * given["x_scale"][rows, None].double()
        t = x @ given["a"][adapter].double().t()
        y[rows] += given["scale"][adapter].double() * (t @ given["b"][adapter].double().t())
    return y

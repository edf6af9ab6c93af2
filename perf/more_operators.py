"""The operators of a worker's residual block as cases to be timed: linear layers with bias,
activation and residual and their gradients, norms around a block's gated and scaled residual
and their gradients, and the clipping of every worker's gradient by its norm.

The n workers' tokens lie one worker after the other in a T x D matrix, and each worker's own
gradient goes into its row of the n x d matrix that the aggregation rules take. ``run()`` does
one operator's pass: through the package where ``own`` is true, else in its plain form, in
elementary torch operations of 32 bits. ``exact()`` is the same in 64 bits, written from the
definitions:

    linear                  p = x w^T + b,  out = act(p) + r
    linear_backward         dx = (dy w) * act'(p) + r
    weight_gradient         dw[w] = sum of dy_t x_t^T, db[w] = sum of dy_t over worker w's tokens
    residual_norm           s = scale x + gate * N_post(h),  y = N(s)
    residual_norm_backward  the gradients of x, h and every parameter, from those of s and y
    clip                    row[w] = min(1, max / |g_w|) g_w, g_w all of worker w's tensors
"""
import math
import random

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
ACTIVATIONS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
EPS = 1e-5
BLOCK = 128  # values that share one exponent in 8-bit blocks


def listed():
    def linear(name, tokens, outputs, inputs, dtype, activation, pre, residual):
        return dict(name=name, kind="linear", tokens=tokens, outputs=outputs, inputs=inputs,
                    dtype=dtype, activation=activation, pre=pre, residual=residual, bias=True)

    def backward(name, tokens, outputs, inputs, dtype, activation, residual):
        return dict(name=name, kind="linear_backward", tokens=tokens, outputs=outputs,
                    inputs=inputs, dtype=dtype, activation=activation, residual=residual)

    def gradient(name, workers, tokens, outputs, inputs, dtype):
        return dict(name=name, kind="weight_gradient", workers=workers, tokens=tokens,
                    outputs=outputs, inputs=inputs, dtype=dtype)

    def norm(name, tokens, width, dtype, rms, post, gate, y8):
        return dict(name=name, kind="residual_norm", tokens=tokens, width=width, dtype=dtype,
                    rms=rms, post=post, gate=gate, y8=y8)

    def norm_backward(name, workers, tokens, width, dtype, rms, post, gate):
        return dict(name=name, kind="residual_norm_backward", workers=workers, tokens=tokens,
                    width=width, dtype=dtype, rms=rms, post=post, gate=gate)

    def clip(name, workers, d, pieces, dtype):
        return dict(name=name, kind="clip", workers=workers, d=d, pieces=pieces, dtype=dtype)

    return [
        # a single token back onto its residual stream: latency and the weights' bytes
        linear("linear_token_4096x4096", 1, 4096, 4096, "bfloat16", "none", False, True),
        # a large batch through a block's widening layer; the backward pass needs p
        linear("linear_16384x8192x2048", 16384, 8192, 2048, "bfloat16", "gelu", True, False),
        # a ragged batch through an odd layer in 32 bits
        backward("linear_backward_777x1000x1500", 777, 1000, 1500, "float32", "relu", True),
        # the large batch back through the narrowing layer to the activation's input
        backward("linear_backward_16384x2048x8192", 16384, 2048, 8192, "bfloat16", "gelu", False),
        # 11 workers with few tokens each, an odd layer: the gradient rows' bytes count
        gradient("weight_gradient_n11_1000x1001x500", 11, 1000, 1001, 500, "float16"),
        # 19 workers' large batches: each worker's product into its row
        gradient("weight_gradient_n19_16384x2048x8192", 19, 16384, 2048, 8192, "bfloat16"),
        # a single token between two blocks, norms on both sides: latency
        norm("residual_norm_token_4096", 1, 4096, "bfloat16", True, True, "columns", False),
        # the largest batch of a training step; the next layer takes the result in 8 bits too
        norm("residual_norm_65536x4096", 65536, 4096, "bfloat16", False, True, "columns", True),
        # 7 workers with few, unequal batches of a small model in 32 bits, of an odd width
        norm_backward("residual_norm_backward_n7_1031x1000", 7, 1031, 1000, "float32", False, True,
                      "columns"),
        # 19 workers' large batches, each token with a gate of its own
        norm_backward("residual_norm_backward_n19_32768x4096", 19, 32768, 4096, "bfloat16", True,
                      True, "tokens"),
        # 11 workers' gradients of a small model, six tensors
        clip("clip_n11_100000", 11, 100_000, 6, "float32"),
        # 19 workers' gradients of a model of 25.6 million values in 161 tensors
        clip("clip_n19_25557032", 19, 25_557_032, 161, "float32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_backward", "weight_gradient", "residual_norm",
                       "residual_norm_backward", "clip"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float32", "float16"])
    if kind in ("residual_norm", "residual_norm_backward"):
        width = _log(rng, 32, 8192)
        if rng.random() < 0.5:
            width = max(32, width // 64 * 64)
        c = dict(kind=kind, tokens=_log(rng, 1, min(65536, (1 << 26) // width)), width=width,
                 dtype=dtype, rms=rng.random() < 0.5, post=rng.random() < 0.7,
                 gate=rng.choice(["none", "columns", "columns", "tokens"]))
        if kind == "residual_norm":
            c["y8"] = rng.random() < 0.4
        else:
            c["workers"] = rng.randint(1, 19)
        return c
    if kind == "clip":
        return dict(kind=kind, workers=rng.randint(1, 19), d=_log(rng, 1000, 25_000_000),
                    pieces=_log(rng, 1, 200), dtype=rng.choice(["float32", "float32", "bfloat16",
                                                                "mixed"]))
    outputs, inputs = _log(rng, 64, 4096), _log(rng, 64, 4096)
    if rng.random() < 0.5:
        outputs, inputs = max(64, outputs // 64 * 64), max(64, inputs // 64 * 64)
    c = dict(kind=kind, outputs=outputs, inputs=inputs, dtype=dtype)
    if kind == "weight_gradient":
        return dict(c, workers=rng.randint(1, 19), tokens=_log(rng, 32, 16384))
    c["tokens"] = _log(rng, 1, 16384)
    c["activation"] = rng.choice(ACTIVATIONS)
    c["residual"] = rng.random() < 0.5
    if kind == "linear":
        c["pre"] = c["activation"] != "none" and rng.random() < 0.5
        c["bias"] = rng.random() < 0.7
    return c


def _counts(case):
    """Tokens of each worker: unequal, their sum the case's tokens."""
    n, t = case["workers"], case["tokens"]
    r = random.Random(n * 1_000_003 + t)
    w = [r.uniform(0.8, 1.2) for _ in range(n)]
    cuts = [int(t * sum(w[:i + 1]) / sum(w)) for i in range(n - 1)] + [t]
    return [b - a for a, b in zip([0] + cuts[:-1], cuts)]


def _lengths(case):
    """Values of each tensor: from a bias's few to a large layer's, their sum d."""
    d, k = case["d"], min(case["pieces"], case["d"])
    r = random.Random(k * 1_000_003 + d)
    w = [math.exp(r.uniform(0.0, 6.0)) for _ in range(k)]
    lengths = [1 + int((d - k) * v / sum(w)) for v in w]
    lengths[-1] += d - sum(lengths)
    return lengths


def _types(case):
    if case["dtype"] != "mixed":
        return [TYPES[case["dtype"]]] * case["pieces"]
    r = random.Random(case["pieces"])
    return [r.choice(list(TYPES.values())) for _ in range(case["pieces"])]


# ---------------------------------------------------------------------------
# Inputs.
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _activations(rows, width, gen):
    """Hidden states: a spread and an offset of each channel, a few channels far larger."""
    x = _normal(gen, rows, width)
    u = torch.rand(width, device="cuda", generator=gen)
    x *= torch.where(u < 0.005, 20.0, 0.5 + u)
    return x.add_(0.3 * _normal(gen, width))


def _gradients(rows, width, gen):
    """Gradients of a loss averaged over a batch: small, some tokens' far larger than others'."""
    return _normal(gen, rows, width).mul_(1e-2 * _normal(gen, rows, 1).exp())


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "clip":  # half of the workers' norms, about, are beyond the maximum
        spread = 1e-3 * _normal(gen, case["workers"], 1).exp()
        s["grads"] = [(_normal(gen, case["workers"], length) * spread).to(t)
                      for length, t in zip(_lengths(case), _types(case))]
        s["max_norm"] = 1e-3 * math.sqrt(case["d"])
        s["rows"] = torch.zeros(case["workers"], case["d"], device="cuda")
        return s
    dtype = TYPES[case["dtype"]]
    if kind in ("linear", "linear_backward", "weight_gradient"):
        t, n, k = case["tokens"], case["outputs"], case["inputs"]
        if kind != "weight_gradient":
            s["w"] = _normal(gen, n, k).mul_(k ** -0.5).to(dtype)
        if kind == "linear":
            s["x"] = _activations(t, k, gen).to(dtype)
            s["bias"] = 0.1 * _normal(gen, n) if case["bias"] else None
            s["residual"] = _activations(t, n, gen).to(dtype) if case["residual"] else None
            return s
        s["dy"] = _gradients(t, n, gen).to(dtype)
        if kind == "linear_backward":
            s["pre"] = None if case["activation"] == "none" else _normal(gen, t, k).to(dtype)
            s["residual"] = _gradients(t, k, gen).to(dtype) if case["residual"] else None
        else:
            s["x"] = _activations(t, k, gen).to(dtype)
            s["counts"] = _counts(case)
            s["grads"] = torch.zeros(case["workers"], n * k + n, device="cuda")
        return s
    t, width, rms = case["tokens"], case["width"], case["rms"]

    def parameter(at, spread):
        return at + spread * _normal(gen, width)

    s["h"] = _activations(t, width, gen).to(dtype)
    s["weight"] = parameter(1, 0.2)
    s["bias"] = None if rms else parameter(0, 0.1)
    s["post_weight"] = parameter(1, 0.2) if case["post"] else None
    s["post_bias"] = parameter(0, 0.1) if case["post"] and not rms else None
    s["gate"] = {"none": lambda: None, "columns": lambda: parameter(0.5, 0.2),
                 "tokens": lambda: torch.rand(t, width, device="cuda", generator=gen).to(dtype)
                 }[case["gate"]]()
    s["scale"] = 0.875
    x = _activations(t, width, gen).to(dtype)
    if kind == "residual_norm":
        s["x"] = x
        return s
    # what the forward pass left
    total, _, stats = _forward(s, x)
    s["s"] = total.to(dtype)
    s["stats"] = stats
    s["ds"] = _gradients(t, width, gen).to(dtype)
    s["dy"] = _gradients(t, width, gen).to(dtype)
    s["counts"] = _counts(case)
    s["grads"] = torch.zeros(case["workers"], len(_parameters(case)) * width, device="cuda")
    return s


def _parameters(case):
    """The parameters with a gradient of each worker, in their order in its row."""
    names = ["weight"] if case["rms"] else ["weight", "bias"]
    if case["post"]:
        names += ["post_weight"] if case["rms"] else ["post_weight", "post_bias"]
    return names + (["gate"] if case["gate"] == "columns" else [])


# ---------------------------------------------------------------------------
# One pass: the package's calls, or the plain form.
def run(s):
    return _calls(s) if own else _plain(s)


def _calls(s):
    import paper_2010_05888_amd as gf

    case = s["case"]
    kind = case["kind"]
    if kind == "clip":
        return [gf.clip_gradients(s["grads"], s["max_norm"], out=s["rows"]), s["rows"]]
    act = None if case.get("activation") in (None, "none") else case["activation"]
    if kind == "linear":
        r = gf.linear(s["x"], s["w"], s["bias"], act, s["residual"], pre=case["pre"])
        return [r.out, r.pre] if case["pre"] else r.out
    if kind == "linear_backward":
        return gf.linear_backward(s["dy"], s["w"], s["pre"], act, s["residual"])
    if kind == "weight_gradient":
        n, k, g = case["outputs"], case["inputs"], s["grads"]
        gf.linear_weight_gradient(s["dy"], s["x"], s["counts"], out=g[:, :n * k].view(-1, n, k),
                                  dbias=g[:, n * k:])
        return g
    rms, scale = case["rms"], s["scale"]
    if kind == "residual_norm":
        r = gf.residual_norm(s["x"], s["h"], s["weight"], s["bias"], s["post_weight"],
                             s["post_bias"], s["gate"], scale, EPS, rms, y8=case["y8"])
        kept = [r.y8.restore(torch.bfloat16)] if case["y8"] else []
        return [r.s, r.y] + [v for v in (r.mean, r.rstd, r.post_mean, r.post_rstd)
                             if v is not None] + kept
    width = case["width"]
    into = {"d" + name: s["grads"][:, i * width:(i + 1) * width]
            for i, name in enumerate(_parameters(case))}
    r = gf.residual_norm_backward(gf.ResidualNorm(s["s"], None, None, *s["stats"]), s["h"],
                                  s["ds"], s["dy"], s["weight"], s["post_weight"], s["post_bias"],
                                  s["gate"], scale, rms, s["counts"], **into)
    return [r.dx, r.dh, s["grads"]] + ([r.dgate] if case["gate"] == "tokens" else [])


def _act(name, p):
    if name == "relu":
        return p.clamp(min=0)
    if name == "gelu":
        return 0.5 * p * (1 + torch.erf(p * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * p * (1 + torch.tanh((2 / math.pi) ** 0.5 * (p + 0.044715 * p * p * p)))
    return p / (1 + torch.exp(-p)) if name == "silu" else p


def _slope(name, p):
    """The activation's derivative; relu's is 0 at 0."""
    if name == "relu":
        return (p > 0).float()
    if name == "gelu":
        density = (2 * math.pi) ** -0.5 * torch.exp(-0.5 * p * p)
        return 0.5 * (1 + torch.erf(p * 0.5 ** 0.5)) + p * density
    if name == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = torch.tanh(c * (p + 0.044715 * p * p * p))
        return 0.5 * (1 + t) + 0.5 * p * (1 - t * t) * c * (1 + 3 * 0.044715 * p * p)
    q = 1 / (1 + torch.exp(-p))
    return q * (1 + p * (1 - q))


def _norm(v, weight, bias, rms):
    """(the norm of v's rows, their mean or None, 1 / deviation)."""
    mean = None if rms else v.mean(1, keepdim=True)
    c = v if rms else v - mean
    rstd = ((c * c).mean(1, keepdim=True) + EPS).rsqrt()
    y = c * rstd * weight
    return (y if bias is None else y + bias), None if rms else mean[:, 0], rstd[:, 0]


def _forward(s, x):
    """(s, y, [mean, rstd, post_mean, post_rstd]) in 32 bits."""
    rms = s["case"]["rms"]
    f, pm, pr = s["h"].float(), None, None
    if s["post_weight"] is not None:
        f, pm, pr = _norm(f, s["post_weight"], s["post_bias"], rms)
    if s["gate"] is not None:
        f = f * s["gate"].float()
    total = s["scale"] * x.float() + f
    y, mean, rstd = _norm(total, s["weight"], s["bias"], rms)
    return total, y, [mean, rstd, pm, pr]


def _norm_gradient(g, hat, rstd, rms):
    """The gradient of a norm's input from that of its normed values."""
    g = g - hat * (g * hat).mean(1, keepdim=True) - (0 if rms else g.mean(1, keepdim=True))
    return rstd[:, None] * g


def _power(s):
    """2^s of whole numbers s from -126 to 127, exactly."""
    return ((s.to(torch.int32) + 127) << 23).view(torch.float32)


def _kept_in_8_bits(x):
    """What the 8-bit blocks of x's rows stand for: 128 values as e4m3 codes times 2^s, the
    smallest s (at least -117) with max |v| <= 448 * 2^s."""
    rows, width = x.shape
    blocks = -(-width // BLOCK)
    v = torch.zeros(rows, blocks * BLOCK, device=x.device)
    v[:, :width] = x
    v = v.view(rows, blocks, BLOCK)
    m, e = torch.frexp(v.abs().amax(2, keepdim=True))
    s = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-117)  # 448 = 0.875 * 2^9
    q = (v * _power(-s)).to(torch.float8_e4m3fn).float()
    return (q * _power(s)).view(rows, -1)[:, :width]


def _of_workers(counts):
    """workers x tokens: 1 where the token is the worker's."""
    n = len(counts)
    w = torch.repeat_interleave(torch.arange(n), torch.tensor(counts)).cuda()
    return (w == torch.arange(n, device="cuda")[:, None]).float()


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "clip":
        square = sum(g.double().square().sum(1) for g in s["grads"])
        norms = square.sqrt()
        factor = (s["max_norm"] / norms).clamp(max=1).float()
        return [norms.float(), torch.cat([g.float() for g in s["grads"]], 1) * factor[:, None]]
    dtype = TYPES[case["dtype"]]
    if kind == "linear":
        p = s["x"].float() @ s["w"].float().T
        p = p if s["bias"] is None else p + s["bias"]
        out = _act(case["activation"], p)
        out = (out if s["residual"] is None else out + s["residual"].float()).to(dtype)
        return [out, p.to(dtype)] if case["pre"] else out
    if kind == "linear_backward":
        dx = s["dy"].float() @ s["w"].float()
        dx = dx if s["pre"] is None else dx * _slope(case["activation"], s["pre"].float())
        return (dx if s["residual"] is None else dx + s["residual"].float()).to(dtype)
    if kind == "weight_gradient":
        # every worker's tokens padded to the longest batch, then one batched product
        counts = torch.tensor(s["counts"])
        at = (counts.cumsum(0) - counts)[:, None] + torch.arange(int(counts.max()))
        mine = (torch.arange(at.shape[1]) < counts[:, None]).cuda()
        at = at.clamp(max=case["tokens"] - 1).cuda()
        dy = torch.where(mine[:, :, None], s["dy"].float()[at], 0.0)
        x = torch.where(mine[:, :, None], s["x"].float()[at], 0.0)
        dw = torch.bmm(dy.transpose(1, 2).contiguous(), x)
        return torch.cat([dw.flatten(1), dy.sum(1)], 1)
    if kind == "residual_norm":
        total, y, stats = _forward(s, s["x"])
        kept = [_kept_in_8_bits(y).to(torch.bfloat16)] if case["y8"] else []
        return [total.to(dtype), y.to(dtype)] + [v for v in stats if v is not None] + kept
    rms = case["rms"]
    mean, rstd, pm, pr = s["stats"]
    total, h, dy = s["s"].float(), s["h"].float(), s["dy"].float()
    hat = (total if rms else total - mean[:, None]) * rstd[:, None]
    g = s["ds"].float() + _norm_gradient(dy * s["weight"], hat, rstd, rms)
    sums = [dy * hat] if rms else [dy * hat, dy]
    gate = None if s["gate"] is None else s["gate"].float()
    df, f = (g if gate is None else g * gate), h
    dh = df
    if case["post"]:
        post = (h if rms else h - pm[:, None]) * pr[:, None]
        f = post * s["post_weight"] + (0 if rms else s["post_bias"])
        sums += [df * post] if rms else [df * post, df]
        dh = _norm_gradient(df * s["post_weight"], post, pr, rms)
    if case["gate"] == "columns":
        sums.append(g * f)
    of = _of_workers(s["counts"])
    out = [(s["scale"] * g).to(dtype), dh.to(dtype), torch.cat([of @ v for v in sums], 1)]
    return out + ([(g * f).to(dtype)] if case["gate"] == "tokens" else [])


# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "clip":
        read = sum(length * t.itemsize for length, t in zip(_lengths(case), _types(case)))
        n, d = case["workers"], case["d"]
        return {"bytes": n * (read + 4 * d + 4), "flops": 3 * n * d}
    size, t = TYPES[case["dtype"]].itemsize, case["tokens"]
    if kind in ("linear", "linear_backward", "weight_gradient"):
        n, k = case["outputs"], case["inputs"]
        if kind == "linear":
            moved = t * k + n * k + t * n * (1 + case["pre"] + case["residual"])
            more = 4 * n if case["bias"] else 0
        elif kind == "linear_backward":
            moved = t * n + n * k + t * k * (1 + (case["activation"] != "none") + case["residual"])
            more = 0
        else:
            moved, more = t * (n + k), 4 * case["workers"] * n * (k + 1)
        return {"bytes": moved * size + more, "flops": 2 * t * n * k}
    width, gate = case["width"], case["gate"]
    stats = 4 * t * (1 if case["rms"] else 2) * (1 + case["post"])
    given = 4 * width * ((1 if case["rms"] else 2) * (1 + case["post"]) + (gate == "columns"))
    if kind == "residual_norm":
        held = t * width + t * -(-width // BLOCK) if case["y8"] else 0
        each = 4 + (gate == "tokens")
        return {"bytes": each * t * width * size + stats + given + held + held * 2,
                "flops": 18 * t * width}
    each = 5 + (case["post"] or gate != "none") + 2 * (gate == "tokens")
    return {"bytes": each * t * width * size + stats + given
            + 4 * case["workers"] * len(_parameters(case)) * width, "flops": 36 * t * width}


# ---------------------------------------------------------------------------
# The definitions in 64 bits.
def _activation(name):
    """The activation and its derivative."""
    def phi(p):
        return torch.special.ndtr(p)

    c, a = math.sqrt(2 / math.pi), 0.044715

    def u(p):  # gelu_tanh is p times the logistic function of this
        return 2 * c * (p + a * p ** 3)

    return {
        "none": (lambda p: p, torch.ones_like),
        "relu": (lambda p: torch.where(p > 0, p, 0), lambda p: torch.where(p > 0, 1.0, 0.0).double()),
        "gelu": (lambda p: p * phi(p),
                 lambda p: phi(p) + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)),
        "gelu_tanh": (lambda p: p * torch.sigmoid(u(p)),
                      lambda p: torch.sigmoid(u(p)) * (1 + p * torch.sigmoid(-u(p))
                                                       * 2 * c * (1 + 3 * a * p ** 2))),
        "silu": (lambda p: p * torch.sigmoid(p),
                 lambda p: torch.sigmoid(p) + p * torch.sigmoid(p) * torch.sigmoid(-p)),
    }[name]


def _statistics(v, rms):
    if rms:
        return torch.zeros_like(v[:, 0]), 1 / torch.sqrt(v.pow(2).sum(1) / v.shape[1] + EPS)
    var, mean = torch.var_mean(v, 1, unbiased=False)
    return mean, 1 / torch.sqrt(var + EPS)


def _e4m3(v):
    """The nearest e4m3 value (3 bits after the leading one, exponents from -6), ties to even."""
    step = torch.exp2(v.abs().clamp(min=2.0 ** -6).log2().floor() - 3)
    return torch.round(v / step) * step


def _kept(x):
    """x as 8-bit blocks give it back."""
    out = torch.empty_like(x)
    for b in range(0, x.shape[1], BLOCK):
        v = x[:, b:b + BLOCK]
        top = v.abs().amax(1, keepdim=True) / 448
        s = top.clamp(min=2.0 ** -117).log2().ceil()
        s = torch.where(torch.exp2(s - 1) >= top, s - 1, s)  # where the logarithm was rounded up
        s = torch.where(torch.exp2(s) < top, s + 1, s).clamp(min=-117)
        out[:, b:b + BLOCK] = _e4m3(v / torch.exp2(s)) * torch.exp2(s)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        g = torch.cat([p.double() for p in s["grads"]], 1)
        norms = torch.linalg.vector_norm(g, dim=1)
        return [norms, g.mul_(torch.where(norms > s["max_norm"], s["max_norm"] / norms,
                                          1.0)[:, None])]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if kind == "linear":
        f, _ = _activation(case["activation"])
        p = torch.mm(d["x"], d["w"].T.contiguous()) + d.get("bias", 0)
        out = f(p) + d.get("residual", 0)
        return [out, p] if case["pre"] else out
    if kind == "linear_backward":
        _, slope = _activation(case["activation"])
        dx = torch.mm(d["dy"], d["w"])
        return (dx * slope(d["pre"]) if "pre" in d else dx) + d.get("residual", 0)
    if kind == "weight_gradient":
        return torch.stack([torch.cat([(a.T @ b).reshape(-1), a.sum(0)])
                            for a, b in zip(d["dy"].split(s["counts"]), d["x"].split(s["counts"]))])
    rms, post, gate, width = case["rms"], case["post"], d.get("gate", 1.0), case["width"]
    if kind == "residual_norm":
        f, stats = d["h"], []
        if post:
            mean, rstd = _statistics(f, rms)
            f = (f - mean[:, None]) * rstd[:, None] * d["post_weight"] + d.get("post_bias", 0)
            stats = [rstd] if rms else [mean, rstd]
        total = s["scale"] * d["x"] + gate * f
        mean, rstd = _statistics(total, rms)
        y = (total - mean[:, None]) * rstd[:, None] * d["weight"] + d.get("bias", 0)
        return [total, y] + ([rstd] if rms else [mean, rstd]) + stats \
            + ([_kept(y)] if case["y8"] else [])
    mean, rstd, pm, pr = (0 if v is None else v.double()[:, None] for v in s["stats"])

    def through(g, z, r):
        """Back through z = (v - mean) * r."""
        along = 0 if rms else g.sum(1, keepdim=True) / width
        return r * (g - along - z * ((g * z).sum(1, keepdim=True) / width))

    z = (d["s"] - mean) * rstd
    g = d["ds"] + through(d["dy"] * d["weight"], z, rstd)
    df = g * gate
    by_name = {"weight": d["dy"] * z, "bias": d["dy"]}
    if post:
        z = (d["h"] - pm) * pr
        by_name.update(post_weight=df * z, post_bias=df)
        f = z * d["post_weight"] + d.get("post_bias", 0)
        dh = through(df * d["post_weight"], z, pr)
    else:
        f, dh = d["h"], df
    by_name["gate"] = g * f
    rows = torch.stack([torch.cat([v[a:a + c].sum(0) for v in (by_name[k] for k in _parameters(case))])
                        for a, c in zip([sum(s["counts"][:i]) for i in range(len(s["counts"]))],
                                        s["counts"])])
    return [s["scale"] * g, dh, rows] + ([by_name["gate"]] if case["gate"] == "tokens" else [])

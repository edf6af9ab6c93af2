"""A worker's operators as cases to be timed: layer norm and its gradient, 8-bit
activation checkpoints, products of 8-bit blocks, and weight gradients.

The n workers' tokens lie one worker after the other in a T x D matrix, and each
worker's own gradient goes into its row of the n x d matrix that the aggregation
rules take. ``run()`` does one operator's pass: through the package where ``own``
is true, else in its plain form, in elementary torch operations of 32 bits.
``exact()`` is the same in 64 bits, written from the definitions.

An 8-bit block is 128 values of a row as e4m3 codes and one exponent s: the
smallest with max |v| <= 448 * 2^s (at least -117), held as s + 127. Rows are
padded with zeros to whole blocks and exponents to multiples of four.
"""
import math
import random

import torch

own = False

BLOCK = 128
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
EPS = 1e-5


def listed():
    def norm(name, tokens, width, dtype, y8=False, x8=False):
        return dict(name=name, kind="norm", tokens=tokens, width=width, dtype=dtype, y8=y8, x8=x8)

    def norm_backward(name, workers, tokens, width, dtype, x8=False):
        return dict(name=name, kind="norm_backward", workers=workers, tokens=tokens, width=width,
                    dtype=dtype, x8=x8)

    def checkpoint(name, rows, width, dtype, transposed=False):
        return dict(name=name, kind="checkpoint", rows=rows, width=width, dtype=dtype,
                    transposed=transposed)

    def linear(name, tokens, outputs, inputs, dtype, out, fast, bias=True):
        return dict(name=name, kind="linear", tokens=tokens, outputs=outputs, inputs=inputs,
                    dtype=dtype, out=out, fast=fast, bias=bias)

    def gradient(name, workers, tokens, outputs, inputs, dtype):
        return dict(name=name, kind="gradient", workers=workers, tokens=tokens, outputs=outputs,
                    inputs=inputs, dtype=dtype)

    return [
        # a single token, answered as it comes: latency
        norm("norm_token_4096", 1, 4096, "bfloat16"),
        # a worker's ordinary batch; the next layer takes the result in 8 bits, so both come out
        norm("norm_8192x2048_y8", 8192, 2048, "bfloat16", y8=True),
        # the largest batch of a training step; its input is kept in 8 bits for the backward pass
        norm("norm_65536x4096_x8", 65536, 4096, "bfloat16", x8=True),
        # 7 workers with few, unequal batches of a small model in 32 bits, of an odd width
        norm_backward("norm_backward_n7_1031x1000", 7, 1031, 1000, "float32"),
        # 19 workers' large batches, the input read from its 8-bit checkpoint
        norm_backward("norm_backward_n19_32768x4096", 19, 32768, 4096, "bfloat16", x8=True),
        # a small activation kept for the backward pass and brought back, of an odd width
        checkpoint("checkpoint_500x1000", 500, 1000, "float16"),
        # a layer's weights after an update, for the input gradient's product
        checkpoint("checkpoint_8192x8192_transposed", 8192, 8192, "bfloat16", True),
        # a single token through a layer: bound by the weights' bytes
        linear("linear_token_4096x4096", 1, 4096, 4096, "bfloat16", "bfloat16", False),
        # a ragged batch through an odd layer, the result in 32 bits
        linear("linear_777x1000x1500", 777, 1000, 1500, "float32", "float32", False),
        # the largest layer and batch, on the 8-bit instruction (its sums are narrower than 32 bits,
        # which 16-bit results hardly show)
        linear("linear_16384x8192x8192", 16384, 8192, 8192, "bfloat16", "bfloat16", True, False),
        # 11 workers with few tokens each, an odd layer: the gradient rows' bytes count
        gradient("gradient_n11_1000x1001x500", 11, 1000, 1001, 500, "float32"),
        # 19 workers' large batches: each worker's product into its row
        gradient("gradient_n19_16384x4096x4096", 19, 16384, 4096, 4096, "bfloat16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "checkpoint", "linear", "linear", "gradient"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float32", "float16"])
    if kind in ("norm", "norm_backward", "checkpoint"):
        width = _log(rng, 32, 8192)
        if rng.random() < 0.5:
            width = max(32, width // 64 * 64)
        rows = _log(rng, 1, min(65536, (1 << 26) // width))
        if kind == "norm":
            return dict(kind=kind, tokens=rows, width=width, dtype=dtype, y8=rng.random() < 0.5,
                        x8=rng.random() < 0.5)
        if kind == "checkpoint":
            return dict(kind=kind, rows=rows, width=width, dtype=dtype,
                        transposed=rng.random() < 0.5)
        return dict(kind=kind, workers=rng.randint(1, 19), tokens=rows, width=width, dtype=dtype,
                    x8=rng.random() < 0.5)
    outputs, inputs = _log(rng, 64, 4096), _log(rng, 64, 4096)
    if rng.random() < 0.5:
        outputs, inputs = max(64, outputs // 64 * 64), max(64, inputs // 64 * 64)
    if kind == "linear":
        out = rng.choice(["bfloat16", "float16", "float32"])
        return dict(kind=kind, tokens=_log(rng, 1, 16384), outputs=outputs, inputs=inputs,
                    dtype=dtype, out=out, fast=out != "float32" and rng.random() < 0.5,
                    bias=rng.random() < 0.5)
    return dict(kind=kind, workers=rng.randint(1, 19), tokens=_log(rng, 32, 16384),
                outputs=outputs, inputs=inputs, dtype=dtype)


def _counts(case):
    """Tokens of each worker: unequal, their sum the case's tokens."""
    n, t = case["workers"], case["tokens"]
    r = random.Random(n * 1_000_003 + t)
    w = [r.uniform(0.8, 1.2) for _ in range(n)]
    cuts = [int(t * sum(w[:i + 1]) / sum(w)) for i in range(n - 1)] + [t]
    return [b - a for a, b in zip([0] + cuts[:-1], cuts)]


# ---------------------------------------------------------------------------
# Inputs.
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(rows, width, gen):
    """Hidden states: a spread and an offset of each channel, a few channels far larger."""
    x = torch.randn(rows, width, device="cuda", generator=gen)
    u = torch.rand(width, device="cuda", generator=gen)
    x *= torch.where(u < 0.005, 20.0, 0.5 + u)
    return x.add_(0.3 * torch.randn(width, device="cuda", generator=gen))


def _gradients(rows, width, gen):
    """Gradients of a loss averaged over a batch: small, some tokens' far larger than others'."""
    g = torch.randn(rows, width, device="cuda", generator=gen)
    return g.mul_(1e-4 * torch.randn(rows, 1, device="cuda", generator=gen).exp())


def _power(s):
    """2^s of whole numbers s from -126 to 127, exactly."""
    return ((s.to(torch.int32) + 127) << 23).view(torch.float32)


def _blocks(x):
    """The 8-bit blocks of the rows of x: codes (rows x padded width) and exponents."""
    rows, width = x.shape
    blocks = -(-width // BLOCK)
    v = torch.zeros(rows, blocks * BLOCK, device=x.device)
    v[:, :width] = x
    v = v.view(rows, blocks, BLOCK)
    fine = v.isfinite()
    m, e = torch.frexp(torch.where(fine, v.abs(), 0.0).amax(2))  # max |v| = m * 2^e, m in [1/2, 1)
    s = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-117)  # 448 = 0.875 * 2^9
    q = (torch.where(fine, v, math.nan) * _power(-s).unsqueeze(2)).to(torch.float8_e4m3fn)
    held = torch.full((rows, -(-blocks // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    held[:, :blocks] = (s + 127).to(torch.uint8)
    return q.view(rows, blocks * BLOCK), held


def _values(q, held, width):
    """What the codes and exponents stand for, in 32 bits."""
    rows, blocks = q.shape[0], q.shape[1] // BLOCK
    p = _power(held[:, :blocks].to(torch.int32) - 127)
    return (q.view(rows, blocks, BLOCK).float() * p.unsqueeze(2)).view(rows, -1)[:, :width]


def prepare(case, seed):
    gen = _generator(seed)
    kind = case["kind"]
    dtype = TYPES[case["dtype"]]
    s = {"case": case}
    if kind in ("norm", "norm_backward"):
        width = case["width"]
        x = _activations(case["tokens"], width, gen).to(dtype)
        s["weight"] = 1 + 0.2 * torch.randn(width, device="cuda", generator=gen)
        if kind == "norm":
            s["x"] = x
            s["bias"] = 0.1 * torch.randn(width, device="cuda", generator=gen)
        else:  # what the forward pass left
            s["dy"] = _gradients(case["tokens"], width, gen).to(dtype)
            s["mean"] = x.float().mean(1)
            s["rstd"] = (x.float().var(1, unbiased=False) + EPS).rsqrt()
            s["counts"] = _counts(case)
            s["x"] = _blocks(x) if case["x8"] else x
            s["grads"] = torch.zeros(case["workers"], 2 * width, device="cuda")
    elif kind == "checkpoint":
        s["x"] = _activations(case["rows"], case["width"], gen).to(dtype)
    elif kind == "linear":
        s["x"] = _activations(case["tokens"], case["inputs"], gen).to(dtype)
        w = torch.randn(case["outputs"], case["inputs"], device="cuda", generator=gen)
        s["w8"] = _blocks(w.mul_(case["inputs"] ** -0.5))
        s["bias"] = 0.1 * torch.randn(case["outputs"], device="cuda", generator=gen) \
            if case["bias"] else None
    else:
        n, k = case["outputs"], case["inputs"]
        s["dy"] = _gradients(case["tokens"], n, gen).to(dtype)
        s["x8"] = _blocks(_activations(case["tokens"], k, gen))
        s["counts"] = _counts(case)
        s["grads"] = torch.zeros(case["workers"], n * k + n, device="cuda")
    return s


# ---------------------------------------------------------------------------
# One pass: the package's calls, or the plain form.
def run(s):
    return _calls(s) if own else _plain(s)


def _calls(s):
    import paper_2010_05888_amd as gf

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        r = gf.layernorm(s["x"], s["weight"], s["bias"], EPS, y8=case["y8"], x8=case["x8"])
        kept = [c.restore(torch.bfloat16) for c in (r.y8, r.x8) if c is not None]
        return [r.y, r.mean, r.rstd] + kept
    if kind == "norm_backward":
        width = case["width"]
        x = gf.Checkpoint(*s["x"], width) if case["x8"] else s["x"]
        g = s["grads"]
        dx, _, _ = gf.layernorm_backward(s["dy"], x, s["mean"], s["rstd"], s["weight"],
                                         s["counts"], dweight=g[:, :width], dbias=g[:, width:])
        return [dx, g]
    if kind == "checkpoint":
        c = gf.checkpoint(s["x"], transposed=case["transposed"])
        return [c.restore(s["x"].dtype), c.exponents]
    if kind == "linear":
        w8 = gf.Checkpoint(*s["w8"], case["inputs"])
        return gf.linear8(gf.checkpoint(s["x"]), w8, s["bias"], TYPES[case["out"]],
                          fast=case["fast"])
    n, k, g = case["outputs"], case["inputs"], s["grads"]
    gf.weight_gradient(s["dy"], gf.Checkpoint(*s["x8"], k), s["counts"],
                       out=g[:, :n * k].view(-1, n, k), dbias=g[:, n * k:])
    return g


def _of_workers(counts):
    """workers x tokens: 1 where the token is the worker's."""
    n = len(counts)
    w = torch.repeat_interleave(torch.arange(n), torch.tensor(counts)).cuda()
    return (w == torch.arange(n, device="cuda")[:, None]).float()


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        c = x - mean
        rstd = ((c * c).mean(1, keepdim=True) + EPS).rsqrt()
        y = c * rstd * s["weight"] + s["bias"]
        kept = [_values(*_blocks(v), case["width"]).to(torch.bfloat16)
                for v, asked in ((y, case["y8"]), (x, case["x8"])) if asked]
        return [y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]] + kept
    if kind == "norm_backward":
        dy = s["dy"].float()
        x = _values(*s["x"], case["width"]) if case["x8"] else s["x"].float()
        xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"]
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True)
                                   - xh * (g * xh).mean(1, keepdim=True))
        of = _of_workers(s["counts"])
        return [dx.to(s["dy"].dtype), torch.cat([of @ (dy * xh), of @ dy], 1)]
    if kind == "checkpoint":
        x = s["x"].float()
        x = x.T if case["transposed"] else x
        q, held = _blocks(x)
        return [_values(q, held, x.shape[1]).to(s["x"].dtype), held]
    if kind == "linear":
        x = _values(*_blocks(s["x"].float()), case["inputs"])
        y = x @ _values(*s["w8"], case["inputs"]).T
        return (y if s["bias"] is None else y + s["bias"]).to(TYPES[case["out"]])
    # every worker's tokens padded to the longest batch, then one batched product
    counts = torch.tensor(s["counts"])
    at = (counts.cumsum(0) - counts)[:, None] + torch.arange(int(counts.max()))
    mine = (torch.arange(at.shape[1]) < counts[:, None]).cuda()
    at = at.clamp(max=case["tokens"] - 1).cuda()
    dy = torch.where(mine[:, :, None], s["dy"].float()[at], 0.0)
    x = torch.where(mine[:, :, None], _values(*s["x8"], case["inputs"])[at], 0.0)
    dw = torch.bmm(dy.transpose(1, 2).contiguous(), x)
    return torch.cat([dw.flatten(1), dy.sum(1)], 1)


# ---------------------------------------------------------------------------
def _held(rows, width):
    """Bytes of the 8-bit blocks of a matrix."""
    return rows * width + rows * -(-width // BLOCK)


def work(case):
    kind = case["kind"]
    size = TYPES[case["dtype"]].itemsize
    if kind in ("norm", "norm_backward"):
        t, width = case["tokens"], case["width"]
        if kind == "norm":
            held = _held(t, width) * (case["y8"] + case["x8"])
            return {"bytes": 2 * t * width * size + 8 * t + 8 * width + held,
                    "flops": 8 * t * width}
        x = _held(t, width) if case["x8"] else t * width * size
        return {"bytes": 2 * t * width * size + x + 8 * t + 4 * width
                + 8 * case["workers"] * width, "flops": 14 * t * width}
    if kind == "checkpoint":
        rows, width = case["rows"], case["width"]
        held = _held(*((width, rows) if case["transposed"] else (rows, width)))
        return {"bytes": 2 * rows * width * size + held, "flops": 3 * rows * width}
    t, n, k = case["tokens"], case["outputs"], case["inputs"]
    if kind == "linear":
        return {"bytes": t * k * size + _held(n, k) + t * n * TYPES[case["out"]].itemsize
                + (4 * n if case["bias"] else 0), "flops": 2 * t * n * k}
    return {"bytes": t * n * size + _held(t, k) + 4 * case["workers"] * n * (k + 1),
            "flops": 2 * t * n * k}


# ---------------------------------------------------------------------------
# The definitions in 64 bits.
def _rounded(v):
    """The nearest e4m3 value (3 bits after the leading one, exponents from -6), ties to even."""
    step = torch.exp2(v.abs().clamp(min=2.0 ** -6).log2().floor() - 3)
    return torch.round(v / step) * step


def _kept(x):
    """x as 8-bit blocks give it back, and the exponents s + 127."""
    rows, width = x.shape
    blocks = -(-width // BLOCK)
    out = torch.empty_like(x)
    held = torch.full((rows, -(-blocks // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    for b in range(blocks):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        top = v.abs().amax(1, keepdim=True) / 448
        s = top.clamp(min=2.0 ** -117).log2().ceil()
        s = torch.where(torch.exp2(s - 1) >= top, s - 1, s)  # where the logarithm was rounded up
        s = torch.where(torch.exp2(s) < top, s + 1, s).clamp(min=-117)
        out[:, b * BLOCK:(b + 1) * BLOCK] = _rounded(v / torch.exp2(s)) * torch.exp2(s)
        held[:, b] = (s[:, 0] + 127).to(torch.uint8)
    return out, held


def _given(blocks, width):
    q, held = blocks
    p = torch.exp2(held.double() - 127).repeat_interleave(BLOCK, 1)
    return q[:, :width].double() * p[:, :width]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = 1 / torch.sqrt(var + EPS)
        y = (x - mean[:, None]) * rstd[:, None] * s["weight"].double() + s["bias"].double()
        kept = [_kept(v)[0] for v, asked in ((y, case["y8"]), (x, case["x8"])) if asked]
        return [y, mean, rstd] + kept
    if kind == "norm_backward":
        dy, mean, rstd, w = (s[k].double() for k in ("dy", "mean", "rstd", "weight"))
        x = _given(s["x"], case["width"]) if case["x8"] else s["x"].double()
        xh = (x - mean[:, None]) * rstd[:, None]
        width = case["width"]
        along = dy @ w / width
        across = (dy * w * xh).sum(1) / width
        dx = (dy * w - along[:, None] - xh * across[:, None]) * rstd[:, None]
        rows = [torch.cat([(a * b).sum(0), a.sum(0)])
                for a, b in zip(dy.split(s["counts"]), xh.split(s["counts"]))]
        return [dx, torch.stack(rows)]
    if kind == "checkpoint":
        x = s["x"].double()
        return list(_kept(x.T.contiguous() if case["transposed"] else x))
    if kind == "linear":
        y = _kept(s["x"].double())[0] @ _given(s["w8"], case["inputs"]).T
        return y if s["bias"] is None else y + s["bias"].double()
    dy, x = s["dy"].double(), _given(s["x8"], case["inputs"])
    return torch.stack([torch.cat([(a.T @ b).reshape(-1), a.sum(0)])
                        for a, b in zip(dy.split(s["counts"]), x.split(s["counts"]))])

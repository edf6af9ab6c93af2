"""The operators of a worker's residual block in 64 bits, from their definitions, with bounds
of what fp32 arithmetic may be off. u = 2^-24."""
import math

import torch

from worker_reference import U

ACTIVATIONS = ["relu", "gelu", "gelu_tanh", "silu"]
TANH, CUBE = 2 * math.sqrt(2 / math.pi), 0.044715
# the largest slope of each activation is 1.13 (gelu's)
STEEPEST = 1.13


def activation(name, p):
    if name is None:
        return p
    if name == "relu":
        return torch.where(p > 0, p, torch.zeros_like(p))
    if name == "gelu":
        return p * torch.special.erfc(-p / math.sqrt(2)) / 2
    if name == "gelu_tanh":
        return p * torch.sigmoid(TANH * (p + CUBE * p ** 3))
    return p * torch.sigmoid(p)


def slope(name, p):
    if name is None:
        return torch.ones_like(p)
    if name == "relu":
        return (p > 0).double()
    if name == "gelu":
        return torch.special.erfc(-p / math.sqrt(2)) / 2 \
            + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        u = TANH * (p + CUBE * p ** 3)
        return torch.sigmoid(u) + p * torch.sigmoid(u) * torch.sigmoid(-u) \
            * TANH * (1 + 3 * CUBE * p ** 2)
    return torch.sigmoid(p) * (1 + p * torch.sigmoid(-p))


def activation_bound(p):
    """An activation evaluated in fp32 at p: a few operations of relative error u on p times a
    factor in [0, 1], whose own argument's rounding moves it by p^2 phi(p) u or less."""
    return 16 * U * (1 + p.abs())


def slope_bound(p):
    """The same of a slope: terms of at most 1.13, their arguments' rounding moves them by |p|^3
    phi(p) u or less, which is below 1.1 u (gelu_tanh's alike, with p (1 + 3 c p^2) for p)."""
    return 32 * U * torch.ones_like(p)


def product(a, b, depth):
    """a b and what fp32 sums of `depth` products may be off: 2 n u of their magnitudes (the
    matrix instructions' adder may cut off where it does not round)."""
    return a @ b, 2 * (depth + 2) * U * (a.abs() @ b.abs())


def linear(x, w, bias, name, residual):
    """(out, its bound), (pre, its bound), before they are rounded to a type."""
    x, w = x.double(), w.double()
    p, off = product(x, w.T.contiguous(), x.shape[1])
    if bias is not None:
        p = p + bias.double()
        off = off + U * p.abs()
    out = activation(name, p)
    bound = off if name is None else STEEPEST * off + activation_bound(p)
    if residual is not None:
        out = out + residual.double()
        bound = bound + U * (out.abs() + bound)
    return (out, bound), (p, off)


def linear_backward(dy, w, pre, name, residual):
    dx, off = product(dy.double(), w.double(), dy.shape[1])
    if name is not None:
        k = slope(name, pre.double())
        off = off * (k.abs() + 1e-6) + dx.abs() * slope_bound(pre.double()) + U * (dx * k).abs()
        dx = dx * k
    if residual is not None:
        dx = dx + residual.double()
        off = off + U * (dx.abs() + off)
    return dx, off


def weight_gradient(dy, x, counts):
    """dw and db of each worker, and their bounds."""
    dy, x = dy.double(), x.double()
    out = []
    for a, b in zip(dy.split(counts), x.split(counts)):
        dw, off = product(a.T.contiguous(), b, len(a))
        out.append((dw, off, a.sum(0), 2 * (len(a) + 2) * U * a.abs().sum(0)))
    return [torch.stack(v) for v in zip(*out)]


# --------------------------------------------------------------------------- norms
def depth(cols):
    """Terms that a lane adds up, and the additions across lanes."""
    return 100.0 + cols / 256


def norm(v, off, weight, bias, eps, rms):
    """The norm of v's rows, v itself off by `off`: (y, bound), (mean, bound), (rstd, bound)."""
    n = depth(v.shape[1])
    mean = torch.zeros_like(v[:, 0]) if rms else v.mean(1)
    c = v - mean[:, None]
    rstd = 1 / torch.sqrt((c * c).mean(1) + eps)
    dmean = torch.zeros_like(mean) if rms else \
        n * U * v.abs().mean(1) + U * mean.abs() + off.mean(1)
    each = off + dmean[:, None] + U * (v.abs() + c.abs())
    dvar = ((2 * c.abs() + each) * each).mean(1) + (n + 3) * U * (c * c).mean(1)
    drel = 0.5 * dvar * rstd ** 2 + 4 * U
    w = weight.double()
    y = c * rstd[:, None] * w + (0 if bias is None else bias.double())
    size = (c * rstd[:, None] * w).abs()
    bound = (w.abs() * rstd[:, None] * each + size * (drel[:, None] + 4 * U) + 2 * U * y.abs()) * 1.01
    return (y, bound + 1e-40), (mean, dmean), (rstd, drel * rstd)


def residual_norm(x, h, weight, bias, post_weight, post_bias, gate, scale, eps, rms):
    """{name: (value, bound)} of s, y and the statistics."""
    x, f = x.double(), h.double()
    off, out = torch.zeros_like(f), {}
    if post_weight is not None:
        (f, off), out["post_mean"], out["post_rstd"] = norm(f, off, post_weight, post_bias, eps, rms)
    g = torch.ones_like(f) if gate is None else gate.double().expand_as(f)
    s = scale * x + g * f
    off = g.abs() * off + 2 * U * ((scale * x).abs() + (g * f).abs())
    out["s"] = (s, off)
    if weight is not None:
        out["y"], out["mean"], out["rstd"] = norm(s, off, weight, bias, eps, rms)
    return out


def _through(g, off, z, weight, rstd, rms):
    """Back through a norm: the gradient of its input and its bound; g is off by `off`, z by 3u."""
    n, weight, rstd = depth(g.shape[1]) + 20, weight.double(), rstd[:, None]
    gw = g * weight
    along = torch.zeros_like(rstd) if rms else gw.mean(1, keepdim=True)
    size = gw.abs() + (0 if rms else gw.abs().mean(1, keepdim=True)) \
        + z.abs() * (gw * z).abs().mean(1, keepdim=True)
    ow = off * weight.abs()
    more = ow + (0 if rms else ow.mean(1, keepdim=True)) + z.abs() * (ow * z.abs()).mean(1, keepdim=True)
    return rstd * (gw - along - z * (gw * z).mean(1, keepdim=True)), rstd * (more + n * U * size) + 1e-44


def residual_norm_backward(ds, dy, s, h, mean, rstd, post_mean, post_rstd, weight, post_weight,
                           post_bias, gate, scale, rms, counts):
    """{name: (value, bound)} of dx, dh, and the parameters' gradients of each worker."""
    h = h.double()
    d = lambda t: None if t is None else t.double()  # noqa: E731
    mean, rstd, post_mean, post_rstd = d(mean), d(rstd), d(post_mean), d(post_rstd)
    g, off = torch.zeros_like(h), torch.zeros_like(h)
    by_token = {}
    if dy is not None:
        z = (s.double() - (0 if rms else mean[:, None])) * rstd[:, None]
        g, off = _through(dy.double(), off, z, weight, rstd, rms)
        by_token["weight"] = (dy.double() * z, 4 * U * (dy.double() * z).abs())
        by_token["bias"] = (dy.double(), torch.zeros_like(g))
    if ds is not None:
        g = g + ds.double()
        off = off + U * (g.abs() + off)
    elif dy is None:
        raise ValueError("no gradient")
    k = torch.ones_like(h) if gate is None else gate.double().expand_as(h)
    df, doff = g * k, off * k.abs() + U * (g * k).abs()
    f, foff = h, torch.zeros_like(h)
    out = {"dx": (scale * g, abs(scale) * off + U * (scale * g).abs()), "dh": (df, doff)}
    if post_weight is not None:
        z = (h - (0 if rms else post_mean[:, None])) * post_rstd[:, None]
        f = z * post_weight.double() + (0 if post_bias is None else post_bias.double())
        foff = 4 * U * ((z * post_weight.double()).abs() + f.abs())
        out["dh"] = _through(df, doff, z, post_weight, post_rstd, rms)
        by_token["post_weight"] = (df * z, doff * z.abs() + 4 * U * (df * z).abs())
        by_token["post_bias"] = (df, doff)
    gf = (g * f, off * f.abs() + g.abs() * foff + off * foff + U * (g * f).abs())
    by_token["gate"] = gf
    out["dgate_by_token"] = gf
    for name, (v, e) in by_token.items():
        out["d" + name] = (torch.stack([p.sum(0) for p in v.split(counts)]),
                           torch.stack([q.sum(0) + (len(p) + 4) * U * p.abs().sum(0) + 1e-44
                                        for p, q in zip(v.split(counts), e.split(counts))]))
    return out


def clip(grads, max_norm):
    """Norms and every worker's row, float64."""
    g = torch.cat([t.detach().cpu().double().reshape(t.shape[0], -1) for t in grads], 1)
    norms = g.pow(2).sum(1).sqrt()
    factor = torch.where(norms <= max_norm, torch.ones_like(norms), max_norm / norms)
    return norms, g * factor[:, None]

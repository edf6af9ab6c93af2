"""The worker's operators in 64 bits on the CPU, from their definitions."""
import torch

BLOCK = 128
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24  # half an fp32 unit in the last place, relative
# half a unit in the last place of a type, relative; and its smallest step's half
HALF = {F32: (2.0 ** -24, 2.0 ** -150), BF16: (2.0 ** -8, 2.0 ** -134), F16: (2.0 ** -11, 2.0 ** -25)}


def shift(top: torch.Tensor) -> torch.Tensor:
    """The smallest s >= -117 with top <= 448 * 2^s (float64 in, float64 out)."""
    m, e = torch.frexp(top)
    return torch.where(top > 0, torch.where(m <= 0.875, e - 9, e - 8), -117).clamp(min=-117).double()


def half_step(v: torch.Tensor) -> torch.Tensor:
    """Half the distance of e4m3 values around v."""
    _, e = torch.frexp(v.abs().clamp(min=2.0 ** -6))
    return torch.exp2(e.double() - 1 - 3 - 1)


def e4m3(v: torch.Tensor) -> torch.Tensor:
    """v (float64) rounded to e4m3 values, ties to even."""
    step = 2 * half_step(v)
    return torch.round(v / step) * step


def blocks(x: torch.Tensor):
    """(values, exponents padded to fours) of x in 8-bit blocks, float64."""
    x = x.double()
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    out = torch.empty_like(x)
    held = torch.full((rows, -(-nb // 4) * 4), 127, dtype=torch.uint8)
    for b in range(nb):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        fine = v.isfinite()
        s = shift(torch.where(fine, v.abs(), 0.0).amax(1))
        p = torch.exp2(s)[:, None]
        q = e4m3(v / p)
        q = torch.where(s[:, None] == 120, q.clamp(-240, 240), q)  # 256 * 2^120 is no fp32 value
        out[:, b * BLOCK:(b + 1) * BLOCK] = torch.where(fine, q * p, float("nan"))
        held[:, b] = (s + 127).to(torch.uint8)
    return out, held


def layernorm(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1 / torch.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None] * weight.double()
    return (y if bias is None else y + bias.double()), mean, rstd


def layernorm_backward(dy, x, mean, rstd, weight, counts):
    """dx, and each worker's dweight and dbias; then the sums of magnitudes that
    their rounding errors are relative to."""
    dy, x, mean, rstd, weight = (t.double() for t in (dy, x, mean, rstd, weight))
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * weight
    gh = (g * h).mean(1, keepdim=True)
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - h * gh)
    size = rstd[:, None] * (g.abs() + g.abs().mean(1, keepdim=True)
                            + h.abs() * (g * h).abs().mean(1, keepdim=True))
    parts = list(zip(dy.split(counts), h.split(counts)))
    dw = torch.stack([(a * b).sum(0) for a, b in parts])
    db = torch.stack([a.sum(0) for a, _ in parts])
    dws = torch.stack([(a * b).abs().sum(0) for a, b in parts])
    dbs = torch.stack([a.abs().sum(0) for a, _ in parts])
    return (dx, dw, db), (size, dws, dbs)


def rounded(ref, dtype):
    """What rounding ref to dtype may add to an error."""
    rel, least = HALF[dtype]
    return ref.abs() * rel + least


def close(got, ref, bound, what=""):
    """|got - ref| <= bound wherever ref is finite; the same NaN and infinities."""
    got, ref = got.double().cpu(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    fine = ref.isfinite()
    assert torch.equal(fine, got.isfinite()), f"{what}: other values are finite"
    assert torch.equal(ref.isnan(), got.isnan()), f"{what}: other values are NaN"
    over = ((got - ref).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: {float(over.max())} beyond the bound at {int(over.argmax())}"

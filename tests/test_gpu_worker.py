"""The worker's operators on the GPU against their definitions in 64 bits.

Tolerances follow from the arithmetic, with u = 2^-24:
* checkpoints: none, a code depends on its block's bits alone;
* sums of n fp32 terms: n u times the sum of the terms' magnitudes (any order);
  on matrix instructions 2 n u, whose adder may cut off where it does not round;
* a result in a type: half a unit in its last place.
"""
import ctypes
import random

import pytest
import torch

import paper_2010_05888_amd as gf
import worker_reference as ref
from worker_reference import BF16, F16, F32, U, close, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [F32, BF16, F16]


@pytest.fixture(scope="module", autouse=True)
def _library():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    gf.load()


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rand(rows, cols, seed, dtype=F32, scale=1.0):
    """Values whose columns and rows differ in size and offset."""
    g = _gen(seed)
    x = torch.randn(rows, cols, generator=g) * (0.2 + 3 * torch.rand(cols, generator=g) ** 4)
    x = x + 0.5 * torch.randn(cols, generator=g)
    return (x * scale * (0.2 + torch.rand(rows, 1, generator=g))).to(dtype)


def _dev(x, layout="plain"):
    """x on the GPU: as it is, with rows further apart, or one element into an allocation;
    what lies between and around holds NaN."""
    if layout == "plain":
        return x.to(DEV)
    rows, cols = x.shape
    ld = cols + (5 if layout == "strided" else 0)
    flat = torch.full((rows * ld + 9,), float("nan"), dtype=x.dtype, device=DEV)
    at = 0 if layout == "strided" else 1
    view = flat[at:at + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(x)
    return view


def _split(rows, n, seed):
    """n counts that add up to rows; one of them is 0 where n > 2."""
    r = random.Random(seed)
    cuts = sorted(r.randint(0, rows) for _ in range(n - 1))
    counts = [b - a for a, b in zip([0] + cuts, cuts + [rows])]
    if n > 2:
        counts[0], counts[1] = 0, counts[0] + counts[1]
    return counts


# --------------------------------------------------------------------------- checkpoints
SIZES = [(1, 1), (1, 127), (3, 128), (2, 129), (5, 511), (64, 512), (7, 1000), (130, 300),
         (257, 2049), (1000, 65), (2, 40000)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_checkpoint_is_exact(rows, cols, dtype, layout, transposed):
    x = _rand(rows, cols, rows + cols, dtype)
    c = gf.checkpoint(_dev(x, layout), transposed=transposed)
    want, held = ref.blocks(x.T if transposed else x)
    assert torch.equal(c.exponents.cpu(), held)
    assert torch.equal(c.restore(F32).cpu().double(), want)
    assert torch.equal(c.restore(BF16).cpu().double(), want)
    assert torch.equal(c.restore(F16).cpu(), want.float().half())
    assert (c.rows, c.cols) == tuple(want.shape)
    pad = c.values[:, c.cols:].view(torch.uint8)
    assert not pad.any()


@pytest.mark.parametrize("transposed", [False, True])
def test_checkpoint_of_extreme_values(transposed):
    """Blocks of zeros, of denormals, next to the largest float; powers of two around every
    binade; infinities and NaN among finite values."""
    big, inf, nan = 3.4028234e38, float("inf"), float("nan")
    rows = [torch.zeros(128), torch.full((128,), 1e-45), torch.full((128,), -1.1754944e-38),
            torch.full((128,), big), torch.linspace(-448, 448, 128),
            torch.full((128,), 448.0), torch.full((128,), 448.00003),
            torch.cat([torch.full((64,), inf), torch.linspace(0, 1, 64)]),
            torch.cat([torch.full((1,), nan), torch.full((127,), -3.0)]),
            torch.full((128,), -inf), torch.full((128,), nan),
            torch.cat([torch.full((1,), big), torch.full((127,), 1e-38)])]
    rows += [2.0 ** k * torch.linspace(-1.9, 1.9, 128) for k in range(-126, 127, 7)]
    x = torch.stack(rows)
    x = x.T.contiguous() if transposed else x
    c = gf.checkpoint(x.to(DEV), transposed=transposed)
    want, held = ref.blocks(x.T if transposed else x)
    assert torch.equal(c.exponents.cpu(), held)
    got = c.restore(F32).cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(), want.nan_to_num())


def test_checkpoint_of_nothing():
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        for transposed in (False, True):
            c = gf.checkpoint(torch.empty(rows, cols, device=DEV), transposed=transposed)
            assert tuple(c.restore().shape) == ((cols, rows) if transposed else (rows, cols))


def test_checkpoint_from_tensors():
    x = _rand(9, 700, 3)
    c = gf.checkpoint(x.to(DEV))
    wide = torch.full((9, 1024), 0x7f, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    wide[:, :768] = c.values
    held = torch.zeros(9, 12, dtype=torch.uint8, device=DEV)
    held[:, :8] = c.exponents
    d = gf.Checkpoint(wide[:, :768], held[:, :8], 700)
    assert torch.equal(d.restore(F32), c.restore(F32))
    for bad in (lambda: gf.Checkpoint(c.values, c.exponents, 800),
                lambda: gf.Checkpoint(c.values[:, :640], c.exponents, 700),
                lambda: gf.Checkpoint(c.values, c.exponents[:, :4], 700),
                lambda: gf.Checkpoint(c.values[1:], c.exponents, 700),
                lambda: gf.Checkpoint(c.values.view(torch.uint8), c.exponents, 700),
                lambda: gf.Checkpoint(wide.flatten()[8:8 + 768 * 9].view(9, 768), c.exponents, 700)):
        with pytest.raises(ValueError):
            bad()


# --------------------------------------------------------------------------- layer norm
def _statistics_bounds(x, mean, rstd):
    """What fp32 sums of up to 80 terms a lane, and a few more across lanes, may be off:
    of the mean absolutely, of 1 / deviation relatively."""
    x = x.double()
    depth = 100.0
    dmean = depth * U * x.abs().mean(1) + U * mean.abs()
    c = (x - mean[:, None]).abs()
    # the mean's error enters the variance squared; the differences' own rounding linearly
    dvar = (dmean ** 2 + 2 * U * (c * (c + x.abs())).mean(1) + (depth + 3) * U * (c * c).mean(1))
    return dmean, 0.5 * dvar * rstd ** 2 + 4 * U


def _norm_bound(x, y, mean, rstd, weight):
    dmean, drel = _statistics_bounds(x, mean, rstd)
    c = (x.double() - mean[:, None]).abs()
    w = weight.double().abs()
    scaled = (c * rstd[:, None]) * w
    return (w * rstd[:, None] * (dmean[:, None] + U * c) + scaled * (drel[:, None] + 4 * U)
            + 2 * U * y.abs()) * 1.01 + 1e-40


NORM_SIZES = [(1, 1), (3, 7), (1, 128), (5, 129), (4, 512), (9, 513), (33, 1000), (2, 1025),
              (70, 2048), (3, 2055), (6, 4096), (5, 5000), (3, 8193), (2, 16385), (2, 40001),
              (2, 65536), (3, 70001)]


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_layernorm(rows, cols, dtype, layout):
    x = _rand(rows, cols, 7 * rows + cols, dtype)
    wtype = F32 if rows % 2 else dtype
    weight = (1 + 0.3 * torch.randn(cols, generator=_gen(1))).to(wtype)
    bias = torch.randn(cols, generator=_gen(2)).to(wtype) if rows != 2 else None
    r = gf.layernorm(_dev(x, layout), weight.to(DEV), None if bias is None else bias.to(DEV), 1e-5,
                     y8=True, x8=True)
    y, mean, rstd = ref.layernorm(x, weight, bias, 1e-5)
    dmean, drel = _statistics_bounds(x, mean, rstd)
    close(r.mean, mean, dmean, "mean")
    close(r.rstd, rstd, drel * rstd, "rstd")
    bound = _norm_bound(x, y, mean, rstd, weight)
    close(r.y, y, bound + rounded(y.abs() + bound, dtype), "y")
    want, held = ref.blocks(x)
    assert torch.equal(r.x8.exponents.cpu(), held)
    assert torch.equal(r.x8.restore(F32).cpu().double(), want)
    # y8: the exponent of a block whose largest value is off by no more than the bound, and codes
    # within half a step of y
    nb = -(-cols // 128)
    for b in range(nb):
        part = slice(b * 128, min(cols, (b + 1) * 128))
        top, off = y[:, part].abs().amax(1), bound[:, part].amax(1)
        s = r.y8.exponents[:, b].cpu().double() - 127
        assert bool(((ref.shift((top - off).clamp(min=0)) <= s) & (s <= ref.shift(top + off))).all())
        p = torch.exp2(s)[:, None]
        step = ref.half_step((y[:, part].abs() + bound[:, part]) / p) * p
        close(r.y8.restore(F32)[:, part], y[:, part], step + bound[:, part], "y8")
    assert bool((r.y8.exponents[:, nb:] == 127).all())
    assert not r.y8.values[:, cols:].view(torch.uint8).any()


def test_layernorm_outputs_are_independent():
    x = _rand(9, 700, 5, BF16).to(DEV)
    w = torch.ones(700, device=DEV)
    full = gf.layernorm(x, w, y8=True, x8=True)
    for y in (False, True):
        for y8 in (False, True):
            for x8 in (False, True):
                r = gf.layernorm(x, w, y=y, y8=y8, x8=x8)
                assert torch.equal(r.mean, full.mean) and torch.equal(r.rstd, full.rstd)
                assert (r.y is None) == (not y) and (r.y8 is None) == (not y8)
                assert (r.x8 is None) == (not x8)
                if y:
                    assert torch.equal(r.y, full.y)
                if y8:
                    assert torch.equal(r.y8.values.view(torch.uint8),
                                       full.y8.values.view(torch.uint8))
                if x8:
                    assert torch.equal(r.x8.values.view(torch.uint8),
                                       full.x8.values.view(torch.uint8))


def test_layernorm_of_constant_rows_and_far_offsets():
    """A constant row has variance 0 and y = bias; a far offset leaves the differences exact."""
    x = torch.full((3, 1000), 4.0)
    x[1] = 1e4 + (torch.arange(1000) % 2)
    x[2] = -1e30
    b = torch.linspace(-1, 1, 1000)
    r = gf.layernorm(x.to(DEV), torch.ones(1000, device=DEV), b.to(DEV), 1e-5)
    assert torch.equal(r.y[0].cpu(), b)
    y, mean, rstd = ref.layernorm(x, torch.ones(1000), b, 1e-5)
    close(r.y[1:2], y[1:2], _norm_bound(x, y, mean, rstd, torch.ones(1000))[1:2], "y")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_layernorm_keeps_what_is_not_finite_in_its_row(bad):
    x = _rand(5, 600, 8, BF16)
    clean = gf.layernorm(x.to(DEV), torch.ones(600, device=DEV), y8=True, x8=True)
    x[2, 17] = bad
    r = gf.layernorm(x.to(DEV), torch.ones(600, device=DEV), y8=True, x8=True)
    keep = [0, 1, 3, 4]
    for a, b in ((r.y, clean.y), (r.mean, clean.mean), (r.rstd, clean.rstd),
                 (r.y8.restore(), clean.y8.restore()), (r.x8.restore(), clean.x8.restore())):
        assert torch.equal(a[keep], b[keep])
    assert bool(r.y[2].isnan().all()) and bool(r.y8.restore()[2].isnan().all())
    assert int(r.x8.restore()[2].isnan().sum()) == 1


# --------------------------------------------------------------------------- its backward pass
BACKWARD_SIZES = [(1, 1, 1), (3, 5, 7), (4, 37, 129), (1, 64, 512), (7, 211, 513), (3, 50, 1000),
                  (2, 9, 2048), (5, 33, 2050), (3, 17, 4096), (2, 12, 5001), (2, 7, 9000),
                  (3, 5, 20001), (19, 3000, 72)]


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,rows,cols", BACKWARD_SIZES)
def test_layernorm_backward(n, rows, cols, dtype, kept, layout):
    x = _rand(rows, cols, n + rows + cols, dtype)
    dy = _rand(rows, cols, rows - cols, dtype, 0.1)
    weight = (1 + 0.3 * torch.randn(cols, generator=_gen(4))).to(dtype if rows % 2 else F32)
    _, mean, rstd = (t.float() for t in ref.layernorm(x, weight, None, 1e-5))
    counts = _split(rows, n, rows)
    x8 = gf.checkpoint(x.to(DEV)) if kept else None
    given = ref.blocks(x)[0] if kept else x
    rows_out = torch.full((n, 2 * cols + 3), float("nan"), device=DEV)
    dx, dw, db = gf.layernorm_backward(_dev(dy, layout), x8 if kept else _dev(x, layout),
                                       mean.to(DEV), rstd.to(DEV), weight.to(DEV), counts,
                                       dweight=rows_out[:, 1:1 + cols],
                                       dbias=rows_out[:, 2 + cols:2 + 2 * cols])
    (rx, rw, rb), (sx, sw, sb) = ref.layernorm_backward(dy, given, mean, rstd, weight, counts)
    # h = (x - mean) rstd is off by 2 u |h|; a lane's sums have at most 16 terms (long rows: cols
    # / 1024), 12 more additions and products follow
    depth = max(16, cols / 1024) + 20
    bound = depth * U * sx + 1e-44
    close(dx, rx, bound + rounded(rx.abs() + bound, dtype), "dx")
    close(dw, rw, (torch.tensor(counts)[:, None] + 4.0) * U * sw + 1e-44, "dweight")
    close(db, rb, (torch.tensor(counts)[:, None] + 4.0) * U * sb + 1e-44, "dbias")
    gaps = rows_out[:, [0, 1 + cols, 2 + 2 * cols]]
    assert bool(gaps.isnan().all()), "written beside the rows"
    again = gf.layernorm_backward(_dev(dy), x8 if kept else _dev(x), mean.to(DEV), rstd.to(DEV),
                                  weight.to(DEV), counts)
    for a, b in zip(again, (dx, dw, db)):
        assert torch.equal(a, b), "other bits from another layout or call"


def test_layernorm_gradient_against_differences():
    """dx, dweight and dbias of sum(dy * layernorm(x)) against central differences in 64 bits: the
    step h leaves h^2 times third derivatives, here below 1e-7 of the gradient's size."""
    rows, cols, h = 4, 24, 1e-4
    x, dy = _rand(rows, cols, 1).double(), _rand(rows, cols, 2).double()
    w = 1 + 0.3 * torch.randn(cols, generator=_gen(3)).double()
    b = torch.randn(cols, generator=_gen(4)).double()
    x, dy, w, b = (t.float().double() for t in (x, dy, w, b))

    def loss(x, w, b, rows=slice(None)):
        return (dy * ref.layernorm(x, w, b, 1e-5)[0])[rows].sum()

    def difference(f, at):
        g = torch.zeros_like(at)
        for i in range(at.numel()):
            e = torch.zeros_like(at).view(-1)
            e[i] = h
            g.view(-1)[i] = (f(at + e.view_as(at)) - f(at - e.view_as(at))) / (2 * h)
        return g

    r = gf.layernorm(x.float().to(DEV), w.float().to(DEV), b.float().to(DEV))
    dx, dw, db = gf.layernorm_backward(dy.float().to(DEV), x.float().to(DEV), r.mean, r.rstd,
                                       w.float().to(DEV), [1, 3])
    parts = [slice(0, 1), slice(1, 4)]
    for got, want in ((dx, difference(lambda v: loss(v, w, b), x)),
                      (dw, torch.stack([difference(lambda v: loss(x, v, b, p), w) for p in parts])),
                      (db, torch.stack([difference(lambda v: loss(x, w, v, p), b) for p in parts]))):
        close(got, want, 2e-5 * want.abs().max() * torch.ones_like(want), "gradient")


def test_layernorm_backward_keeps_what_is_not_finite_with_its_worker():
    x, dy = _rand(40, 300, 1), _rand(40, 300, 2)
    mean, rstd, w = x.mean(1), torch.ones(40), torch.ones(300)
    counts = [10, 0, 25, 5]

    def call():
        return gf.layernorm_backward(dy.to(DEV), x.to(DEV), mean.to(DEV), rstd.to(DEV), w.to(DEV),
                                     counts)

    clean = call()
    dy[12, 5], x[20, 7] = float("inf"), float("nan")
    dx, dw, db = call()
    rows = [t for t in range(40) if t not in (12, 20)]
    assert torch.equal(dx[rows], clean[0][rows])
    for got, was in ((dw, clean[1]), (db, clean[2])):
        assert torch.equal(got[[0, 1, 3]], was[[0, 1, 3]])
        assert not bool(got[1].any())
    assert bool(dw[2, 7].isnan()) and bool(db[2, 5].isinf()) and bool(dw[2, 8].isfinite())
    assert bool(dx[20].isnan().all())


def test_layernorm_backward_of_nothing():
    e = torch.empty(0, 300, device=DEV)
    v = torch.empty(0, device=DEV)
    dx, dw, db = gf.layernorm_backward(e, e, v, v, torch.ones(300, device=DEV), [0, 0])
    assert dx.shape == (0, 300) and not bool(dw.any()) and not bool(db.any())
    assert dw.shape == db.shape == (2, 300)


# --------------------------------------------------------------------------- products
LINEAR_SIZES = [(1, 1, 1), (1, 16, 128), (1, 100, 1000), (2, 5, 129), (3, 64, 4096), (15, 33, 700),
                (16, 1000, 384), (17, 256, 512), (33, 130, 1500), (64, 64, 64), (100, 77, 2000),
                (128, 128, 256), (129, 257, 640), (200, 300, 1000), (257, 511, 130), (1, 513, 9000),
                (300, 1024, 1024), (600, 520, 128)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("m,n,k", LINEAR_SIZES)
def test_linear8(m, n, k, biased, dtype):
    x, w = _rand(m, k, m + n + k), _rand(n, k, m - n - k, scale=k ** -0.5)
    b = torch.randn(n, generator=_gen(5)) if biased else None
    out = gf.linear8(gf.checkpoint(x.to(DEV)), gf.checkpoint(w.to(DEV)),
                     None if b is None else b.to(DEV), dtype)
    xv, wv = ref.blocks(x)[0], ref.blocks(w)[0]
    want = xv @ wv.T + (0 if b is None else b.double())
    bound = 2 * (k + 4) * U * (xv.abs() @ wv.abs().T + (0 if b is None else b.double().abs()))
    close(out, want, bound + rounded(want.abs() + bound, dtype), "out")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", LINEAR_SIZES)
def test_linear8_fast(m, n, k, dtype):
    """Of every eight products the instruction drops what is below 2^-13 of the largest one's
    binade: at most 8 * 2^-13 of the largest, so 2^-10 of the sum of their magnitudes."""
    x, w = _rand(m, k, m + n + k), _rand(n, k, m - n - k, scale=k ** -0.5)
    b = torch.randn(n, generator=_gen(5))
    out = gf.linear8(gf.checkpoint(x.to(DEV)), gf.checkpoint(w.to(DEV)), b.to(DEV), dtype, fast=True)
    xv, wv = ref.blocks(x)[0], ref.blocks(w)[0]
    want = xv @ wv.T + b.double()
    bound = (2.0 ** -10 + 2 * (k + 4) * U) * (xv.abs() @ wv.abs().T + b.double().abs())
    close(out, want, bound + rounded(want.abs() + bound, dtype), "out")


def test_linear8_against_wide_exponents():
    """Blocks whose exponents differ by far: the products' exponents are added, not lost."""
    m, n, k = 40, 70, 1280
    x, w = _rand(m, k, 1), _rand(n, k, 2)
    for b in range(k // 128):
        x[:, b * 128:(b + 1) * 128] *= 2.0 ** (30 - 6 * b)
        w[:, b * 128:(b + 1) * 128] *= 2.0 ** (6 * b - 30)
    out = gf.linear8(gf.checkpoint(x.to(DEV)), gf.checkpoint(w.to(DEV)), dtype=F32)
    xv, wv = ref.blocks(x)[0], ref.blocks(w)[0]
    close(out, xv @ wv.T, 2 * (k + 4) * U * (xv.abs() @ wv.abs().T), "out")


@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("m", [3, 40, 300])
def test_linear8_keeps_what_is_not_finite_with_its_token(m, fast):
    n, k = 200, 700
    x, w = _rand(m, k, 1), _rand(n, k, 2)
    clean = gf.linear8(gf.checkpoint(x.to(DEV)), gf.checkpoint(w.to(DEV)), fast=fast)
    x[1, 650], w[9, 3] = float("inf"), float("nan")
    out = gf.linear8(gf.checkpoint(x.to(DEV)), gf.checkpoint(w.to(DEV)), fast=fast)
    hit = torch.zeros(m, n, dtype=torch.bool)
    hit[1] = hit[:, 9] = True
    # the blocks of the infinity and the NaN lose one value, which may change their exponents
    assert torch.equal(out.cpu().isnan(), hit)
    assert torch.equal(out.cpu()[~hit], clean.cpu()[~hit])


def test_linear8_of_nothing():
    def c(rows, cols):
        return gf.checkpoint(torch.ones(rows, cols, device=DEV))

    assert gf.linear8(c(0, 100), c(5, 100)).shape == (0, 5)
    assert gf.linear8(c(5, 100), c(0, 100)).shape == (5, 0)
    b = torch.arange(7.0, device=DEV)
    for fast in (False, True):
        assert torch.equal(gf.linear8(c(3, 0), c(7, 0), b, F32, fast), b.expand(3, 7))


# --------------------------------------------------------------------------- weight gradients
GRADIENT_SIZES = [(1, 1, 1, 1), (3, 5, 7, 9), (2, 64, 64, 64), (4, 37, 129, 200), (1, 300, 64, 500),
                  (7, 211, 100, 130), (3, 129, 257, 256), (11, 400, 33, 1000), (2, 1000, 300, 270),
                  (64, 100, 20, 30), (1, 1, 500, 600), (19, 640, 128, 128)]


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,tokens,outputs,inputs", GRADIENT_SIZES)
def test_weight_gradient(n, tokens, outputs, inputs, dtype, layout):
    dy = _rand(tokens, outputs, n + tokens, dtype, 0.01)
    x = _rand(tokens, inputs, n - tokens)
    counts = _split(tokens, n, outputs)
    flat = torch.full((n, outputs * inputs + outputs + 2), float("nan"), device=DEV)
    dw, db = gf.weight_gradient(
        _dev(dy, layout), gf.checkpoint(x.to(DEV)), counts,
        out=flat[:, 1:1 + outputs * inputs].view(n, outputs, inputs),
        dbias=flat[:, 1 + outputs * inputs:-1])
    xv = ref.blocks(x)[0]
    d = dy.double()
    pairs = list(zip(d.split(counts), xv.split(counts)))
    want = torch.stack([a.T @ b for a, b in pairs])
    size = torch.stack([a.abs().T @ b.abs() for a, b in pairs])
    terms = torch.tensor(counts, dtype=torch.float64)[:, None, None] * {F32: 3, F16: 2, BF16: 1}[dtype]
    close(dw, want, 2 * (terms + 4) * U * size + 1e-40, "dw")
    close(db, torch.stack([a.sum(0) for a, _ in pairs]),
          (torch.tensor(counts)[:, None] + 4.0) * U * torch.stack([a.abs().sum(0) for a, _ in pairs])
          + 1e-40, "dbias")
    assert bool(flat[:, [0, -1]].isnan().all()), "written beside the rows"
    again, _ = gf.weight_gradient(_dev(dy), gf.checkpoint(x.to(DEV)), counts)
    assert torch.equal(again, dw), "other bits from another layout or call"


def test_weight_gradient_against_differences():
    """The gradient of sum(dout * linear(x, w)), which is linear in w: differences are exact but for
    rounding (fp64 sums of 60 terms over a step of 1)."""
    tokens, outputs, inputs = 12, 6, 10
    x8 = gf.checkpoint(_rand(tokens, inputs, 1).to(DEV))
    xv = x8.restore(F32).cpu().double()
    dout = _rand(tokens, outputs, 2, BF16)
    dw, _ = gf.weight_gradient(dout.to(DEV), x8, [5, 7])
    w = _rand(outputs, inputs, 3).double()
    for worker, part in enumerate((slice(0, 5), slice(5, 12))):
        want = torch.zeros(outputs, inputs, dtype=torch.float64)
        for i in range(w.numel()):
            e = torch.zeros(w.numel(), dtype=torch.float64)
            e[i] = 0.5
            hi, lo = ((dout.double() * (xv @ (w + s * e.view_as(w)).T))[part].sum() for s in (1, -1))
            want.view(-1)[i] = hi - lo
        close(dw[worker], want, 1e-5 * want.abs().max() * torch.ones_like(want), "dw")


@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient_keeps_what_is_not_finite_with_its_worker(dtype):
    tokens, outputs, inputs = 200, 150, 140
    counts = [70, 0, 61, 69]
    dy, x = _rand(tokens, outputs, 1, dtype), _rand(tokens, inputs, 2)
    clean, _ = gf.weight_gradient(dy.to(DEV), gf.checkpoint(x.to(DEV)), counts)
    dy[75, 3], x[130, 4] = float("inf"), float("nan")
    dw, _ = gf.weight_gradient(dy.to(DEV), gf.checkpoint(x.to(DEV)), counts)
    assert torch.equal(dw[[0, 1, 3]], clean[[0, 1, 3]]) and not bool(dw[1].any())
    hit = torch.zeros(outputs, inputs, dtype=torch.bool)
    hit[3] = hit[:, 4] = True
    assert torch.equal(~dw[2].cpu().isfinite(), hit)
    assert int(dw[2].isinf().sum()) == inputs - 1


def test_weight_gradient_of_largest_values():
    """fp32 values next to the largest and infinities survive their split into bf16 parts."""
    dy = torch.zeros(3, 4)
    dy[0], dy[1, 1], dy[1, 2] = 3.4028234e38, float("inf"), -float("inf")
    x = torch.zeros(3, 8)
    x[0], x[1] = 0.5, 1.0
    dw, _ = gf.weight_gradient(dy.to(DEV), gf.checkpoint(x.to(DEV)))
    want = torch.tensor([3.4028234e38 / 2, float("inf"), -float("inf"), 3.4028234e38 / 2])
    assert torch.equal(dw[0].cpu(), want[:, None].expand(4, 8))


def test_weight_gradient_of_nothing():
    dw, db = gf.weight_gradient(torch.empty(0, 5, device=DEV), gf.checkpoint(torch.empty(0, 9, device=DEV)),
                                [0, 0], dbias=torch.ones(2, 5, device=DEV))
    assert dw.shape == (2, 5, 9) and not bool(dw.any()) and not bool(db.any())
    dw, _ = gf.weight_gradient(torch.ones(4, 5, device=DEV), gf.checkpoint(torch.empty(4, 0, device=DEV)))
    assert dw.shape == (1, 5, 0)


# --------------------------------------------------------------------------- calls
def _everything(t):
    r = gf.layernorm(t["x"], t["w"], t["b"], y8=True, x8=True)
    out = gf.linear8(r.y8, gf.checkpoint(t["v"]))
    dw, db = gf.weight_gradient(t["dout"], r.y8, t["counts"], dbias=torch.empty(3, 300, device=DEV))
    dy = gf.linear8(gf.checkpoint(t["dout"]), gf.checkpoint(t["v"], transposed=True))
    return [r.y, out, dw, db, dy, *gf.layernorm_backward(dy, r.x8, r.mean, r.rstd, t["w"], t["counts"])]


def _inputs(seed):
    return {"x": _rand(400, 1000, seed, BF16).to(DEV), "v": _rand(300, 1000, seed + 1, BF16).to(DEV),
            "dout": _rand(400, 300, seed + 2, BF16, 0.01).to(DEV), "w": torch.ones(1000, device=DEV),
            "b": torch.zeros(1000, device=DEV), "counts": [150, 110, 140]}


def test_calls_run_on_the_current_stream():
    """Two streams at once, each with its own inputs; nothing is shared between their calls."""
    sets = [_inputs(10), _inputs(20)]
    want = [_everything(t) for t in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(_everything(sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for rep in got[i]:
            for a, b in zip(rep, want[i]):
                assert torch.equal(a, b)


def test_calls_in_a_graph():
    t = _inputs(30)
    others = [_inputs(40 + i) for i in range(3)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _everything(t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _everything(t)
    for o in others + others[:1]:
        for k in ("x", "v", "dout"):
            t[k].copy_(o[k])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, _everything(o)):
            assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    """Rows more than 2^31 elements (and 4 GiB) apart."""
    ld, rows, cols = (1 << 31) + 8, 3, 300
    flat = torch.empty(2 * ld + cols, dtype=BF16, device=DEV)
    far = flat.as_strided((rows, cols), (ld, 1))
    x = _rand(rows, cols, 9, BF16)
    far.copy_(x)
    near = x.to(DEV)
    w = torch.ones(cols, device=DEV)
    a, b = (gf.layernorm(t, w, y8=True) for t in (far, near))
    assert torch.equal(a.y, b.y) and torch.equal(a.mean, b.mean)
    for transposed in (False, True):
        assert torch.equal(gf.checkpoint(far, transposed).restore(), gf.checkpoint(near, transposed).restore())
    for got, want in zip(*(gf.layernorm_backward(t, t, b.mean, b.rstd, w, [1, 2]) for t in (far, near))):
        assert torch.equal(got, want)
    x8 = gf.checkpoint(near)
    for got, want in zip(*(gf.weight_gradient(t, x8, [2, 1], dbias=torch.empty(2, cols, device=DEV))
                           for t in (far, near))):
        assert torch.equal(got, want)


def test_refusals():
    x, v = torch.ones(4, 200, device=DEV), torch.ones(200, device=DEV)
    s = torch.ones(4, device=DEV)
    c = gf.checkpoint(x)
    for call in (lambda: gf.checkpoint(x.double()), lambda: gf.checkpoint(v),
                 lambda: gf.checkpoint(x.T), lambda: gf.checkpoint(x[:, ::2]),
                 lambda: gf.checkpoint(v.expand(4, 200)),
                 lambda: c.restore(torch.float64),
                 lambda: gf.layernorm(x, v[:100]), lambda: gf.layernorm(x, v.bfloat16()),
                 lambda: gf.layernorm(x, v, v.double()), lambda: gf.layernorm(x, v.cpu()),
                 lambda: gf.layernorm_backward(x, x.bfloat16(), s, s, v),
                 lambda: gf.layernorm_backward(x, x[:3], s, s, v),
                 lambda: gf.layernorm_backward(x, x, s[:3], s, v),
                 lambda: gf.layernorm_backward(x, x, s, s, v, [1, 2]),
                 lambda: gf.layernorm_backward(x, x, s, s, v, [5, -1]),
                 lambda: gf.layernorm_backward(x, x, s, s, v, []),
                 lambda: gf.layernorm_backward(x, x, s, s, v, dweight=x),
                 lambda: gf.layernorm_backward(x, x, s, s, v, [2, 2], dbias=x[:2, ::2]),
                 lambda: gf.linear8(c, gf.checkpoint(x[:, :100])),
                 lambda: gf.linear8(c, c, v), lambda: gf.linear8(c, c, dtype=torch.int8),
                 lambda: gf.weight_gradient(x[:3], c), lambda: gf.weight_gradient(x, x),
                 lambda: gf.weight_gradient(x, c, [3]),
                 lambda: gf.weight_gradient(x, c, out=torch.empty(1, 200, 100, device=DEV)),
                 lambda: gf.weight_gradient(x, c, [2, 2], dbias=v.expand(2, 200))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gf.layernorm(x, v, eps=-1.0),
                 lambda: gf.layernorm(x[:, :0], v[:0])):
        with pytest.raises(gf.GarfieldError):
            call()
    with pytest.raises(gf.GarfieldError) as e:
        gf.weight_gradient(x, c, [0] * 64 + [4])
    assert e.value.code == gf.ETOOBIG

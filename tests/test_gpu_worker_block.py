"""The operators of a worker's residual block on the GPU against their definitions in 64 bits:
linear layers with their epilogue and gradients, norms around the residual, clipping by norm.

Tolerances (block_reference.py) follow from the arithmetic, with u = 2^-24: sums of n products
on matrix instructions 2 n u of their magnitudes, activations and norms what their few operations
may be off, a result in a type half a unit in its last place.
"""
import ctypes
import math

import pytest
import torch

import paper_2010_05888_amd as gf
from paper_2010_05888_amd import worker
import block_reference as ref
from test_gpu_worker import _dev, _gen, _rand, _split
from worker_reference import BF16, F16, F32, U, close, rounded
import worker_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [F32, BF16, F16]


@pytest.fixture(scope="module", autouse=True)
def _library():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    gf.load()


def _check(got, want, dtype, what):
    value, bound = want
    close(got, value, bound + rounded(value.abs() + bound, dtype), what)


def _maybe(t, to=DEV):
    return None if t is None else t.to(to)


# --------------------------------------------------------------------------- linear layers
LINEAR = [(1, 1, 1), (1, 130, 70), (2, 9, 0), (3, 7, 5), (5, 64, 64), (16, 48, 96), (17, 33, 65),
          (31, 1000, 200), (33, 72, 1000), (64, 128, 256), (65, 200, 129), (130, 70, 1003),
          (257, 263, 520)]


def _layer(m, n, k, dtype, biased=True, residual=True):
    x, w = _rand(m, k, m + n + k, dtype), _rand(n, k, m * n, dtype, max(k, 1) ** -0.5)
    bias = torch.randn(n, generator=_gen(n)).to(F32 if m % 2 else dtype) if biased else None
    return x, w, bias, _rand(m, n, k + 1, dtype) if residual else None


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", LINEAR)
def test_linear(m, n, k, dtype, layout):
    for i, name in enumerate([None] + ref.ACTIVATIONS):
        x, w, bias, residual = _layer(m, n, k, dtype, i != 1, i % 2 == 0)
        r = gf.linear(_dev(x, layout), _dev(w, layout), _maybe(bias), name,
                      None if residual is None else _dev(residual, layout), pre=i != 2)
        out, pre = ref.linear(x, w, bias, name, residual)
        _check(r.out, out, dtype, f"out, {name}")
        if i != 2:
            _check(r.pre, pre, dtype, f"pre, {name}")
        else:
            assert r.pre is None


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", LINEAR)
def test_linear_backward(m, n, k, dtype, layout):
    """m tokens, k outputs (what is added up) and n inputs."""
    for i, name in enumerate([None] + ref.ACTIVATIONS):
        dy, w = _rand(m, k, m + n, dtype, 0.1), _rand(k, n, n + k, dtype, max(k, 1) ** -0.5)
        pre = None if name is None else _rand(m, n, 5, dtype)
        residual = _rand(m, n, 6, dtype, 0.1) if i % 2 else None
        dx = gf.linear_backward(_dev(dy, layout), _dev(w, layout),
                                None if pre is None else _dev(pre, layout), name,
                                None if residual is None else _dev(residual, layout))
        _check(dx, ref.linear_backward(dy, w, pre, name, residual), dtype, f"dx, {name}")


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,tokens,outputs,inputs",
                         [(1, 1, 1, 1), (1, 5, 3, 7), (3, 40, 10, 129), (2, 33, 130, 64),
                          (5, 300, 72, 200), (3, 2, 65, 257), (1, 1000, 64, 128), (19, 190, 33, 65),
                          (2, 513, 264, 136)])
def test_linear_weight_gradient(n, tokens, outputs, inputs, dtype, layout):
    x, dy = _rand(tokens, inputs, 1 + tokens, dtype), _rand(tokens, outputs, 2 + outputs, dtype, 0.1)
    counts = _split(tokens, n, tokens)
    rows = torch.full((n, outputs * inputs + outputs + 3), float("nan"), device=DEV)
    length = outputs * inputs
    gf.linear_weight_gradient(_dev(dy, layout), _dev(x, layout), counts,
                              out=rows[:, 1:1 + length].view(n, outputs, inputs),
                              dbias=rows[:, 2 + length:-1])
    dw, dw_off, db, db_off = ref.weight_gradient(dy, x, counts)
    close(rows[:, 1:1 + length].view(n, outputs, inputs), dw, dw_off + rounded(dw, F32), "dw")
    close(rows[:, 2 + length:-1], db, db_off + rounded(db, F32), "db")
    assert bool(rows[:, [0, 1 + length, -1]].isnan().all()), "written beside the rows"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_activation_backward(name, dtype):
    for rows, cols, layout in ((1, 1, "plain"), (3, 1001, "strided"), (70, 256, "offset"), (5, 4096, "plain")):
        dy = _rand(rows, cols, 1, dtype)
        pre = _rand(rows, cols, 2, dtype, 3.0)
        k = ref.slope(name, pre.double())
        want = dy.double() * k
        off = dy.double().abs() * ref.slope_bound(pre.double()) + U * want.abs()
        _check(gf.activation_backward(_dev(dy, layout), _dev(pre, layout), name), (want, off), dtype, name)


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_activations_at_the_edges(name):
    """From far below to far above 0, where an exponential or a cube passes fp32's range."""
    p = torch.tensor([-3e38, -1e20, -1e13, -200.0, -104.0, -88.5, -20.0, -6.0, -1e-3, -1e-30, 0.0,
                      1e-30, 1e-3, 6.0, 20.0, 88.5, 104.0, 200.0, 1e13, 1e20, 3e38])[None, :]
    k = p.shape[1]
    out = gf.linear(p.to(DEV), torch.eye(k, device=DEV), None, name).out
    want = ref.activation(name, p.double())
    want = torch.where(want.isfinite(), want, torch.where(p > 0, p, 0).double())  # p * 0 far below
    # a factor below 2^-126 is no normal fp32 value and becomes 0: |p| 2^-126 where there is one,
    # which is for |p| < 105
    small = torch.where(p.abs() < 105, p.abs() * 2.0 ** -126, 0.0).double()
    close(out, want, 16 * U * want.abs() + 16 * U * (p.abs() < 30) + small + 1e-40, "value")
    k = ref.slope(name, p.double())
    k = torch.where(k.isfinite(), k, (p > 0).double())
    got = gf.activation_backward(torch.ones_like(p).to(DEV), p.to(DEV), name)
    close(got, k, 32 * U * torch.ones_like(k), "slope")
    nan = torch.full((1, 8), float("nan"), device=DEV)
    assert bool(gf.linear(nan, torch.eye(8, device=DEV), None, name).out.isnan().all())
    if name != "relu":  # whose slope is 0 but for p > 0
        assert bool(gf.activation_backward(torch.ones_like(nan), nan, name).isnan().all())


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_activations_all_along(name):
    """Every 2^-9 from -16 to 16, in fp32, and gelu's small values relative to themselves."""
    p = torch.arange(-16 * 512, 16 * 512 + 1, dtype=torch.float32).mul_(2.0 ** -9)[None, :]
    p = p[:, :p.shape[1] // 64 * 64].reshape(-1, 64)
    out = gf.linear(p.to(DEV), torch.eye(64, device=DEV), None, name).out
    want = ref.activation(name, p.double())
    close(out, want, ref.activation_bound(p.double()), "value")
    if name != "relu":
        part = (p > -6) & (p < -0.01)
        off = ((out.double().cpu() - want) / want)[part].abs().max()
        assert float(off) < 2.0 ** -12, float(off)
    k = ref.slope(name, p.double())
    got = gf.activation_backward(torch.ones_like(p).to(DEV), p.to(DEV), name)
    close(got, k, ref.slope_bound(p.double()), "slope")


@pytest.mark.parametrize("m", [1, 40, 300])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_keeps_what_is_not_finite_with_its_token(m, dtype):
    x, w, bias, residual = _layer(m, 70, 200, dtype)
    clean = gf.linear(x.to(DEV), w.to(DEV), bias.to(DEV), "relu", residual.to(DEV), pre=True)
    at = m // 2
    x[at, 3] = float("nan")
    if m > 2:
        x[at + 1, 5] = float("inf")
        residual[0, 2] = -float("inf")
    r = gf.linear(x.to(DEV), w.to(DEV), bias.to(DEV), "relu", residual.to(DEV), pre=True)
    keep = [t for t in range(m) if t not in (at, at + 1)]
    assert torch.equal(r.pre[keep], clean.pre[keep])
    assert bool(r.pre[at].isnan().all()) and bool(r.out[at].isnan().all())
    if m > 2:
        want = (x[at + 1].double() @ w.double().T).sign() * float("inf")
        assert torch.equal(r.pre[at + 1].double().cpu(), want)
        assert float(r.out[0, 2]) == -float("inf")
        assert torch.equal(r.out[keep[1:]], clean.out[keep[1:]])


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_weight_gradient_keeps_what_is_not_finite_with_its_worker(dtype):
    x, dy = _rand(90, 100, 1, dtype), _rand(90, 60, 2, dtype)
    counts = [30, 0, 41, 19]
    clean = gf.linear_weight_gradient(dy.to(DEV), x.to(DEV), counts)[0]
    x[35, 7], dy[29, 3] = float("nan"), float("inf")
    dw = gf.linear_weight_gradient(dy.to(DEV), x.to(DEV), counts)[0]
    assert torch.equal(dw[[1, 3]], clean[[1, 3]]) and not bool(dw[1].any())
    rows = [j for j in range(60) if j != 3]
    assert torch.equal(dw[0, rows], clean[0, rows]) and not bool(dw[0, 3].isfinite().any())
    cols = [k for k in range(100) if k != 7]
    assert torch.equal(dw[2][:, cols], clean[2][:, cols]) and bool(dw[2, :, 7].isnan().all())


def test_products_of_subnormal_and_largest_values():
    """fp16 values below 2^-14 count, fp32 and bf16 ones next to the largest stay finite."""
    x = torch.full((40, 64), 2.0 ** -24, dtype=F16)
    w = torch.full((8, 64), 1024.0, dtype=F16)
    got = gf.linear(x.to(DEV), w.to(DEV)).out
    assert torch.equal(got.cpu(), torch.full((40, 8), 64 * 2.0 ** -14, dtype=F16))
    for dtype in (F32, BF16):  # subnormal factors of a normal product, in tiles and for few rows
        for rows in (3, 40):
            x = torch.full((rows, 64), 2.0 ** -130, dtype=dtype)
            got = gf.linear(x.to(DEV), w.to(dtype).to(DEV)).out
            assert torch.equal(got.cpu(), torch.full((rows, 8), 2.0 ** -114, dtype=dtype))
    for dtype in (F32, BF16):
        top = torch.finfo(dtype).max
        x = torch.zeros(40, 64, dtype=dtype)
        x[:, 3] = top
        w = torch.zeros(8, 64, dtype=dtype)
        w[:, 3] = 1
        assert torch.equal(gf.linear(x.to(DEV), w.to(DEV)).out.cpu(),
                           torch.full((40, 8), top, dtype=dtype))


def test_linear_of_nothing():
    x, w = torch.empty(0, 9, device=DEV), torch.ones(5, 9, device=DEV)
    assert gf.linear(x, w, pre=True).out.shape == (0, 5)
    assert gf.linear(torch.ones(4, 9, device=DEV), w[:0]).out.shape == (4, 0)
    assert gf.linear_backward(torch.ones(4, 0, device=DEV), w[:0]).tolist() == [[0.0] * 9] * 4
    dw, db = gf.linear_weight_gradient(torch.empty(0, 5, device=DEV), x, [0, 0],
                                       dbias=torch.ones(2, 5, device=DEV))
    assert dw.shape == (2, 5, 9) and not bool(dw.any()) and not bool(db.any())
    dw, db = gf.linear_weight_gradient(torch.ones(4, 5, device=DEV), torch.empty(4, 0, device=DEV),
                                       [1, 3], dbias=torch.zeros(2, 5, device=DEV))
    assert dw.shape == (2, 5, 0) and db.tolist() == [[1.0] * 5, [3.0] * 5]
    assert gf.activation_backward(x, x, "gelu").shape == (0, 9)


def test_linear_gradients_against_differences():
    """Of sum(dout * linear(gelu(linear(x)))): dx and both weights' gradients against central
    differences in 64 bits; the step leaves its square times third derivatives."""
    g = _gen(3)
    x, w1, w2, dout = (torch.randn(*s, generator=g) for s in ((5, 6), (7, 6), (4, 7), (5, 4)))

    def loss(x, w1, w2):
        return (dout.double() * (ref.activation("gelu", x @ w1.T) @ w2.T + x[:, :4])).sum()

    def difference(i):
        at = [x.double(), w1.double(), w2.double()]
        out = torch.zeros_like(at[i])
        for j in range(out.numel()):
            ends = []
            for h in (1e-4, -1e-4):
                moved = [t.clone() for t in at]
                moved[i].view(-1)[j] += h
                ends.append(loss(*moved))
            out.view(-1)[j] = (ends[0] - ends[1]) / 2e-4
        return out

    x_, w1_, w2_, d_ = (t.to(DEV) for t in (x, w1, w2, dout))
    first = gf.linear(x_, w1_, None, "gelu", pre=True)
    dp = gf.linear_backward(d_, w2_, first.pre, "gelu")
    through = torch.zeros(5, 6, device=DEV)
    through[:, :4] = d_
    got = [gf.linear_backward(dp, w1_, residual=through), gf.linear_weight_gradient(dp, x_)[0][0],
           gf.linear_weight_gradient(d_, first.out)[0][0]]
    assert torch.equal(dp, gf.activation_backward(gf.linear_backward(d_, w2_), first.pre, "gelu"))
    for i in range(3):
        want = difference(i)
        close(got[i], want, 2e-5 * want.abs().max() * torch.ones_like(want), str(i))


def test_outputs_with_rows_apart():
    """The C entries write matrices whose rows lie apart, and nothing between them."""
    fn, m, n, k = worker._functions(), 37, 50, 64
    x, w, bias, residual = (t.to(DEV) for t in _layer(m, n, k, BF16))
    wide = torch.full((3, m, n + 6), float("nan"), dtype=BF16, device=DEV)
    stream = torch.cuda.current_stream().cuda_stream
    need = fn["garfield_linear_workspace"](x.data_ptr(), 1, m, k, k, w.data_ptr(), n, k)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    assert fn["garfield_linear"](x.data_ptr(), 1, m, k, k, w.data_ptr(), n, k, bias.data_ptr(), 0, 2,
                                 residual.data_ptr(), n, wide[0].data_ptr(), n + 6,
                                 wide[1].data_ptr(), n + 6, ws.data_ptr(), need, stream) == gf.OK
    r = gf.linear(x, w, bias, "gelu", residual, pre=True)
    assert torch.equal(wide[0, :, :n], r.out) and torch.equal(wide[1, :, :n], r.pre)
    assert fn["garfield_activation_backward"](x.data_ptr(), 1, m, n, k, 2, r.pre.data_ptr(), n,
                                              wide[2].data_ptr(), n + 6, stream) == gf.OK
    assert torch.equal(wide[2, :, :n], gf.activation_backward(x[:, :n], r.pre, "gelu"))
    assert bool(wide[:, :, n:].isnan().all())


# --------------------------------------------------------------------------- norms
NORMS = [(1, 1), (3, 7), (1, 128), (5, 129), (4, 512), (9, 513), (33, 1000), (2, 1025), (70, 2048),
         (3, 2055), (6, 4096), (5, 5000), (3, 8193), (2, 16385), (2, 40001)]
FORMS = [dict(), dict(rms=True, gate=None), dict(post=False), dict(gate="tokens"), dict(norm=False),
         dict(rms=True, gate="tokens", post=False), dict(gate=None, post=False, norm=False),
         dict(norm=False, gate="tokens", rms=True)]


def _block(rows, cols, dtype, rms=False, post=True, gate="columns", norm=True, biased=True):
    wtype = F32 if rows % 2 else dtype

    def vector(at, seed):
        return (at + 0.3 * torch.randn(cols, generator=_gen(seed))).to(wtype)

    return {"weight": vector(1, 1) if norm else None,
            "bias": vector(0, 2) if norm and not rms and biased else None,
            "post_weight": vector(1, 3) if post else None,
            "post_bias": vector(0, 4) if post and not rms and biased else None,
            "gate": {None: None, "columns": vector(0.5, 5),
                     "tokens": _rand(rows, cols, 6, dtype)}[gate]}


def _moved(block, layout="plain"):
    return {k: None if v is None else (_dev(v, layout) if v.dim() == 2 else v.to(DEV))
            for k, v in block.items()}


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", NORMS)
def test_residual_norm(rows, cols, dtype, layout):
    for i, form in enumerate(FORMS):
        block, rms = _block(rows, cols, dtype, biased=i != 3, **form), form.get("rms", False)
        x, h = _rand(rows, cols, rows + cols, dtype), _rand(rows, cols, rows * cols + i, dtype)
        scale, normed = (1.0, 0.7, -1.5)[i % 3], block["weight"] is not None
        r = gf.residual_norm(_dev(x, layout), _dev(h, layout), **_moved(block, layout), scale=scale,
                             rms=rms, y8=normed)
        want = ref.residual_norm(x, h, **block, scale=torch.tensor(scale).double(), eps=1e-5, rms=rms)
        what = f"{form}"
        _check(r.s, want["s"], dtype, "s " + what)
        for name in ("mean", "rstd", "post_mean", "post_rstd"):
            got = getattr(r, name)
            if name not in want or (rms and "mean" in name):
                assert got is None
            else:
                _check(got, want[name], F32, name + what)
        if not normed:
            assert r.y is None and r.y8 is None
            continue
        _check(r.y, want["y"], dtype, "y " + what)
        y, bound = want["y"]
        nb = -(-cols // 128)
        for b in range(nb):  # as layernorm's y8: an exponent within the bound, codes half a step off
            part = slice(b * 128, min(cols, (b + 1) * 128))
            top, off = y[:, part].abs().amax(1), bound[:, part].amax(1)
            s = r.y8.exponents[:, b].cpu().double() - 127
            assert bool(((worker_reference.shift((top - off).clamp(min=0)) <= s)
                         & (s <= worker_reference.shift(top + off))).all())
            p = torch.exp2(s)[:, None]
            step = worker_reference.half_step((y[:, part].abs() + bound[:, part]) / p) * p
            close(r.y8.restore(F32)[:, part], y[:, part], step + bound[:, part], "y8")
        assert bool((r.y8.exponents[:, nb:] == 127).all())
        assert not r.y8.values[:, cols:].view(torch.uint8).any()


def test_residual_norm_outputs_are_independent():
    x, h = _rand(9, 700, 5, BF16).to(DEV), _rand(9, 700, 6, BF16).to(DEV)
    block = _moved(_block(9, 700, BF16))
    full = gf.residual_norm(x, h, **block, y8=True)
    for y, y8 in ((False, False), (False, True), (True, False)):
        r = gf.residual_norm(x, h, **block, y=y, y8=y8)
        assert torch.equal(r.s, full.s) and torch.equal(r.rstd, full.rstd)
        assert (r.y is None) == (not y) and (r.y8 is None) == (not y8)
        assert not y or torch.equal(r.y, full.y)
        assert not y8 or torch.equal(r.y8.values.view(torch.uint8), full.y8.values.view(torch.uint8))


def test_residual_norm_is_layernorm_without_a_block():
    """With h = 0 the stream passes, and y is layernorm()'s to the statistics' rounding."""
    x = _rand(40, 900, 3, BF16).to(DEV)
    w, b = (1 + 0.1 * torch.randn(900, generator=_gen(1))).to(DEV), torch.randn(900, generator=_gen(2)).to(DEV)
    r = gf.residual_norm(x, torch.zeros_like(x), w, b)
    want = gf.layernorm(x, w, b)
    assert torch.equal(r.s, x)
    # layernorm()'s lanes add up to 16 differences d of two values in fp32, each addition off by u of
    # the sum of |d| or less: 15 u mean |d| <= 32 u mean |x| for each side
    close(r.mean, want.mean.cpu(), 64 * U * x.double().abs().mean(1).cpu())
    close(r.y, want.y.cpu(), 2.0 ** -7 * want.y.cpu().double().abs() + 1e-5)


def test_residual_norm_of_rows_far_from_zero():
    """A far offset leaves the differences nearly exact; equal values have variance 0."""
    x = torch.full((2, 1000), 1e4)
    x[1] += torch.arange(1000) % 2
    h = torch.zeros(2, 1000)
    b = torch.linspace(-1, 1, 1000)
    r = gf.residual_norm(x.to(DEV), h.to(DEV), torch.ones(1000, device=DEV), b.to(DEV))
    assert torch.equal(r.y[0].cpu(), b)
    want = worker_reference.layernorm(x, torch.ones(1000), b, 1e-5)[0]
    close(r.y[1:], want[1:], 1e-5 * torch.ones(1, 1000, dtype=torch.float64))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["x", "h"])
def test_residual_norm_keeps_what_is_not_finite_in_its_row(bad, where):
    x, h = _rand(5, 600, 8, BF16), _rand(5, 600, 9, BF16)
    block = _moved(_block(5, 600, BF16))
    clean = gf.residual_norm(x.to(DEV), h.to(DEV), **block, y8=True)
    (x if where == "x" else h)[2, 17] = bad
    r = gf.residual_norm(x.to(DEV), h.to(DEV), **block, y8=True)
    keep = [0, 1, 3, 4]
    for a, b in ((r.s, clean.s), (r.y, clean.y), (r.rstd, clean.rstd), (r.y8.restore(), clean.y8.restore())):
        assert torch.equal(a[keep], b[keep])
    assert bool(r.y[2].isnan().all())


BACKWARD = [(1, 1, 1), (3, 5, 7), (4, 37, 129), (1, 64, 512), (7, 211, 513), (3, 50, 1000),
            (2, 9, 2048), (5, 33, 2050), (3, 17, 4096), (2, 12, 5001), (2, 7, 9000), (3, 5, 20001),
            (19, 3000, 72), (2, 0, 40)]


@pytest.mark.parametrize("layout", ["plain", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,rows,cols", BACKWARD)
def test_residual_norm_backward(n, rows, cols, dtype, layout):
    for i, form in enumerate(FORMS):
        block, rms = _block(rows, cols, dtype, biased=i != 3, **form), form.get("rms", False)
        h, s = _rand(rows, cols, rows + cols, dtype), _rand(rows, cols, rows * cols + i, dtype)
        normed, scale = block["weight"] is not None, (1.0, 0.7, -1.5)[i % 3]
        dy = _rand(rows, cols, 11, dtype, 0.1) if normed else None
        ds = _rand(rows, cols, 12, dtype, 0.1) if i != 2 else None
        ones = torch.ones(cols)
        (_, (mean, _), (rstd, _)) = ref.norm(s.double(), torch.zeros(rows, cols).double(), ones, None, 1e-5, rms)
        (_, (pm, _), (pr, _)) = ref.norm(h.double(), torch.zeros(rows, cols).double(), ones, None, 1e-5, rms)
        stats = [None if rms or not normed else mean.float(), rstd.float() if normed else None,
                 None if rms or block["post_weight"] is None else pm.float(),
                 pr.float() if block["post_weight"] is not None else None]
        counts = _split(rows, n, rows)
        bias = block.pop("bias")
        names = [k for k in ("weight", "bias", "post_weight", "post_bias", "gate")
                 if (k in ("weight", "bias") and normed and not (rms and k == "bias"))
                 or (k == "post_weight" and block[k] is not None)
                 or (k == "post_bias" and block["post_weight"] is not None and not rms)
                 or (k == "gate" and block[k] is not None and block[k].dim() == 1)]
        del bias
        given = torch.full((n, len(names) * (cols + 1) + 1), float("nan"), device=DEV)
        into = {"d" + k: given[:, 1 + j * (cols + 1):(j + 1) * (cols + 1)] for j, k in enumerate(names)}

        def call(layout, **into):
            r = gf.ResidualNorm(_dev(s, layout), None, None, *[_maybe(v) for v in stats])
            return gf.residual_norm_backward(
                r, _dev(h, layout), None if ds is None else _dev(ds, layout),
                None if dy is None else _dev(dy, layout), **_moved(block, layout), scale=scale,
                rms=rms, counts=counts, **into)

        got = call(layout, **into)
        want = ref.residual_norm_backward(ds, dy, s, h, *stats, **block, scale=float(torch.tensor(scale)),
                                          rms=rms, counts=counts)
        _check(got.dx, want["dx"], dtype, f"dx {form}")
        _check(got.dh, want["dh"], dtype, f"dh {form}")
        for k in ("weight", "bias", "post_weight", "post_bias", "gate"):
            v = getattr(got, "d" + k)
            if k in names:
                _check(v, want["d" + k], F32, f"d{k} {form}")
            elif k == "gate" and block["gate"] is not None:
                _check(v, want["dgate_by_token"], dtype, f"dgate {form}")
            else:
                assert v is None
        assert bool(given[:, ::cols + 1].isnan().all()), "written beside the rows"
        if i == 0:
            again = call("plain")
            for a, b in zip(again, got):
                assert torch.equal(a, b), "other bits from another layout or call"


def test_residual_norm_gradients_against_differences():
    """Of sum(ds * s + dy * y) against central differences in 64 bits, each worker's parameters."""
    rows, cols, counts, h0 = 4, 24, [1, 3], 1e-4
    g = _gen(7)
    at = {k: torch.randn(*((rows, cols) if k in ("x", "h") else (cols,)), generator=g).double().float().double()
          for k in ("x", "h", "weight", "bias", "post_weight", "post_bias", "gate")}
    ds, dy = (torch.randn(rows, cols, generator=g) for _ in range(2))
    for rms in (False, True):
        keys = [k for k in at if not (rms and "bias" in k)]

        def loss(v, part):
            out = ref.residual_norm(**{k: v.get(k) for k in at}, scale=0.75, eps=1e-5, rms=rms)
            return (ds.double() * out["s"][0] + dy.double() * out["y"][0])[part].sum()

        def difference(k, part):
            v = {i: at[i] for i in keys}
            out = torch.zeros_like(at[k])
            for j in range(out.numel()):
                ends = []
                for step in (h0, -h0):
                    moved = at[k].clone()
                    moved.view(-1)[j] += step
                    ends.append(loss({**v, k: moved}, part))
                out.view(-1)[j] = (ends[0] - ends[1]) / (2 * h0)
            return out

        dev = {k: at[k].float().to(DEV) for k in keys}
        r = gf.residual_norm(**dev, scale=0.75, rms=rms)
        got = gf.residual_norm_backward(r, dev["h"], ds.to(DEV), dy.to(DEV), dev["weight"],
                                        dev["post_weight"], dev.get("post_bias"), dev["gate"], 0.75,
                                        rms, counts)
        parts = [slice(0, 1), slice(1, 4)]
        for k in keys:
            want = difference(k, slice(None)) if k in ("x", "h") else \
                torch.stack([difference(k, p) for p in parts])
            close(getattr(got, "d" + k), want, 3e-5 * want.abs().max() * torch.ones_like(want), k)


@pytest.mark.parametrize("cols", [300, 5000, 9000])
def test_residual_norm_backward_from_one_gradient(cols):
    """Without dy the norm after passes nothing on and its weight's gradient is 0; without ds the
    rest is as with a ds of zeros."""
    rows, counts = 12, [5, 7]
    s, h, g = (_rand(rows, cols, i).to(DEV) for i in range(3))
    block = _moved(_block(rows, cols, F32))
    block.pop("bias")
    stats = [0.1 * torch.ones(rows, device=DEV), torch.ones(rows, device=DEV)] * 2
    r = gf.ResidualNorm(s, None, None, *stats)

    def call(ds, dy):
        return gf.residual_norm_backward(r, h, ds, dy, **block, counts=counts)

    for a, b in ((call(g, None), call(g, torch.zeros_like(g))), (call(None, g), call(torch.zeros_like(g), g))):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
    assert not bool(call(g, None).dweight.any()) and torch.equal(call(g, None).dx, g)


def test_residual_norm_backward_keeps_what_is_not_finite_with_its_worker():
    rows, cols, counts = 40, 300, [10, 0, 25, 5]
    s, h, ds, dy = (_rand(rows, cols, i) for i in range(4))
    block = _moved(_block(rows, cols, F32))
    block.pop("bias")
    stats = [torch.ones(rows, device=DEV)] * 4

    def call():
        return gf.residual_norm_backward(gf.ResidualNorm(s.to(DEV), None, None, *stats), h.to(DEV),
                                         ds.to(DEV), dy.to(DEV), **block, counts=counts)

    clean = call()
    ds[12, 5], h[20, 7] = float("inf"), float("nan")
    got = call()
    keep = [t for t in range(rows) if t not in (12, 20)]
    for a, b in zip(got, clean):
        if a.shape[0] == rows:
            assert torch.equal(a[keep], b[keep])
        else:
            assert torch.equal(a[[0, 1, 3]], b[[0, 1, 3]]) and not bool(a[1].any())


# --------------------------------------------------------------------------- clipping
def _pieces(n, lengths, types, seed, spread=1.0):
    size = torch.exp(spread * torch.randn(n, 1, generator=_gen(seed)))
    return [(torch.randn(n, k, generator=_gen(seed + i)) * size).to(types[i % len(types)])
            for i, k in enumerate(lengths)]


def _clip_close(got, want, dtype):
    """The factor is rounded once and its product once, then to dtype."""
    close(got, want, 2.02 * U * want.abs() + rounded(want, dtype) + 1e-45, "clipped")


@pytest.mark.parametrize("types", [[F32], [BF16], [F16, F32, BF16]])
@pytest.mark.parametrize("n,lengths", [(1, [1]), (1, [70000]), (3, [1, 0, 17]), (11, [1000, 7, 130, 65, 9]),
                                       (19, [40000, 3, 16384, 16385]), (64, [33, 5]),
                                       (2, [1 + 37 * i for i in range(150)]), (5, [300_001, 8]),
                                       (3, [5] * 100), (2, [131072]), (2, [131072, 1]),
                                       (1, [70_000] * 64), (1, [70_000] * 65), (4, [513, 511, 512])])
def test_clip_gradients(n, lengths, types):
    grads = _pieces(n, lengths, types, n + len(lengths))
    norms = ref.clip(grads, 1.0)[0]
    limit = float(torch.tensor(float(norms.median()) * 0.9).float())  # some are clipped
    norms, rows = ref.clip(grads, limit)
    d = sum(lengths)
    here = [g.to(DEV) for g in grads]
    close(gf.gradient_norms(here), norms, 1.01 * U * norms, "norms")
    wide = torch.full((n, d + 4), float("nan"), device=DEV)
    close(gf.clip_gradients(here, limit, out=wide[:, 1:1 + d]), norms, 1.01 * U * norms, "norms")
    _clip_close(wide[:, 1:1 + d], rows, F32)
    assert bool(wide[:, 0].isnan().all()) and bool(wide[:, 1 + d:].isnan().all())
    for g, was in zip(here, grads):
        assert torch.equal(g.cpu(), was)
    gf.clip_gradients(here, limit)
    at = 0
    for g, was in zip(here, grads):
        _clip_close(g, rows[:, at:at + was.shape[1]], was.dtype)
        at += was.shape[1]
    kept = norms <= limit
    for g, was in zip(here, grads):
        assert torch.equal(g[kept].cpu(), was[kept])


def test_clip_columns_of_one_matrix_and_shapes():
    n = 5
    m = torch.randn(n, 1000, generator=_gen(1)).to(DEV)
    norms, rows = ref.clip([m], 20.0)
    parts = [m[:, 300:900].view(n, 20, 30), m[:, :300], m[:, 950:], m[:, 900:950].view(n, 50)]
    got = gf.clip_gradients(parts, 20.0)
    close(got, norms, 1.01 * U * norms)
    _clip_close(m, rows, F32)


def test_clip_refuses_tensors_that_share_memory():
    m = torch.ones(4, 100, device=DEV)
    for parts in ([m, m], [m[:, :60], m[:, 50:]], [m[:, :50], m[1:, :50].expand(3, 50)],
                  [m.view(400)[None], m.view(400)[None, 399:]]):
        if parts[0].shape[0] != parts[1].shape[0]:
            with pytest.raises(ValueError):
                gf.clip_gradients(parts, 1.0)
            continue
        with pytest.raises(gf.GarfieldError):
            gf.clip_gradients(parts, 1.0)
        assert bool((m == 1).all())
    # nor may the rows that are written, but for columns of the same matrix beside them
    wide = torch.ones(4, 200, device=DEV)
    for parts, out in (([wide[:, :100]], wide[:, :100]), ([wide[:, :60], wide[:, 160:]], wide[:, 50:150]),
                       ([wide.view(1, 800)[:, :200]], wide.view(1, 800)[:, 199:399])):
        with pytest.raises(gf.GarfieldError):
            gf.clip_gradients(parts, 1.0, out=out)
    gf.clip_gradients([wide[:, :60], wide[:, 160:]], 1.0, out=wide[:, 60:160])
    close(wide[:, 60:160], torch.full((4, 100), 0.1), torch.full((4, 100), 2 * U * 0.1))
    assert gf.gradient_norms([m, m]).tolist() == pytest.approx([math.sqrt(200)] * 4)  # reading is fine


def test_clip_of_extreme_values():
    """Sums of squares beyond fp32's range, zeros, and what is not finite."""
    g = torch.zeros(6, 300)
    g[0], g[1], g[3, 7], g[4, 9], g[5] = 3e38, 1e-30, float("inf"), float("nan"), 1.0
    norms, rows = ref.clip([g], 1.0)
    out = torch.empty(6, 300, device=DEV)
    got = gf.clip_gradients(g.to(DEV), 1.0, out=out)
    want = norms.clone()
    want[0] = float("inf")  # 3e38 sqrt(300)
    close(got, want, 1.01 * U * want)
    _clip_close(out[[0, 1, 2, 5]], rows[[0, 1, 2, 5]], F32)
    assert float(out[3, 0]) == 0 and bool(out[3, 7].isnan()) and int(out[3].isnan().sum()) == 1
    assert bool(out[4].isnan().all())
    close(gf.clip_gradients(g.to(DEV), float("inf"), out=out), got.cpu(), torch.zeros(6))
    finite = [0, 1, 2, 5]
    assert torch.equal(out[finite].cpu(), g[finite])
    gf.clip_gradients(g.to(DEV), 0.0, out=out)
    assert not bool(out[finite].any())


# --------------------------------------------------------------------------- calls
def _inputs(seed, dtype=BF16):
    t = {"x": _rand(400, 512, seed, dtype), "h": _rand(400, 512, seed + 1, dtype),
         "w1": _rand(700, 512, seed + 2, dtype, 0.05), "w2": _rand(512, 700, seed + 3, dtype, 0.05),
         "dout": _rand(400, 512, seed + 4, dtype, 0.01), "gain": 1 + 0.1 * _rand(1, 512, seed + 5)[0],
         "gate": 0.5 + 0.1 * _rand(1, 512, seed + 6)[0]}
    return {k: v.to(DEV) for k, v in t.items()}


COUNTS = [150, 110, 0, 140]


def _everything(t):
    """A residual block of a worker, forward and back, and its gradients clipped into rows."""
    r = gf.residual_norm(t["x"], t["h"], t["gain"], post_weight=t["gain"], gate=t["gate"], rms=True)
    up = gf.linear(r.y, t["w1"], None, "gelu", pre=True)
    out = gf.linear(up.out, t["w2"], None, None, r.s)
    dp = gf.linear_backward(t["dout"], t["w2"], up.pre, "gelu")
    dw2, _ = gf.linear_weight_gradient(t["dout"], up.out, COUNTS)
    dw1, _ = gf.linear_weight_gradient(dp, r.y, COUNTS)
    dy = gf.linear_backward(dp, t["w1"])
    b = gf.residual_norm_backward(r, t["h"], t["dout"], dy, t["gain"], t["gain"], None, t["gate"], 1.0,
                                  True, COUNTS)
    rows = torch.empty(4, dw1[0].numel() + dw2[0].numel() + 1536, device=DEV)
    norms = gf.clip_gradients([dw1, dw2, b.dweight, b.dpost_weight, b.dgate], 0.5, out=rows)
    return [r.s, r.y, up.out, up.pre, out.out, dp, dy, b.dx, b.dh, norms, rows]


def test_a_block_is_its_operators_one_after_the_other():
    """The whole run against 64 bits: rows of gradients of the same block by autograd. 16-bit steps
    between the operators cost half a unit each, 2^-8 of a value; a dozen of them at random stay
    below 2% of a gradient's size."""
    t = _inputs(50)
    got = _everything(t)
    d = {k: v.double().cpu().requires_grad_() for k, v in t.items()}
    first = [0, 150, 260, 260, 400]
    for worker_ in (0, 1, 3):
        part = slice(first[worker_], first[worker_ + 1])
        out = ref.residual_norm(d["x"][part], d["h"][part], d["gain"], None, d["gain"].detach(), None,
                                d["gate"], 1.0, 1e-5, True)
        s, y = out["s"][0], out["y"][0]
        z = ref.activation("gelu", y @ d["w1"].T) @ d["w2"].T + s
        gain, gate, w1, w2, x, h = torch.autograd.grad(
            (d["dout"].detach()[part] * z).sum(),
            [d["gain"], d["gate"], d["w1"], d["w2"], d["x"], d["h"]])
        rows = got[10][worker_].double().cpu()
        norm = float(got[9][worker_])
        scale = max(1.0, norm / 0.5)
        n1, n2 = w1.numel(), w2.numel()
        for want, have in ((w1, rows[:n1] * scale), (w2, rows[n1:n1 + n2] * scale),
                           (gain, rows[n1 + n2:n1 + n2 + 512] * scale),
                           (gate, rows[-512:] * scale)):
            off = float((have.view_as(want) - want).norm() / want.norm())
            assert off < 0.02, off
        for want, have in ((x[part], got[7][part]), (h[part], got[8][part])):
            assert float((have.double().cpu() - want).norm() / want.norm()) < 0.02
    assert not bool(got[10][2].any()) and float(got[9][2]) == 0


def test_calls_run_on_the_current_stream():
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
    others = [_inputs(40 + 10 * i) for i in range(3)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _everything(t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _everything(t)
    for o in others + others[:1]:
        for k in t:
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
    near, w = x.to(DEV), _rand(40, cols, 3, BF16).to(DEV)
    gain = torch.ones(cols, device=DEV)

    def call(v):
        r = gf.residual_norm(v, v, gain, post_weight=gain, gate=v)
        b = gf.residual_norm_backward(r, v, v, v, gain, gain, None, v, counts=[1, 2])
        rows = torch.empty(3, cols, device=DEV)
        return [r.s, r.y, *b, gf.linear(v, w).out, gf.linear(w, v).out, gf.linear(w, v, pre=True).pre,
                gf.linear_backward(near[:, :3].contiguous(), v, v, "silu", v),
                *gf.linear_weight_gradient(v, v, [2, 1], dbias=torch.empty(2, cols, device=DEV)),
                gf.activation_backward(v, v, "gelu"), gf.clip_gradients(v, 1.0, out=rows), rows]

    for a, b in zip(call(far), call(near)):
        assert (a is None and b is None) or torch.equal(a, b)


def test_refusals():
    x, v = torch.ones(4, 200, device=DEV), torch.ones(200, device=DEV)
    w, s = torch.ones(7, 200, device=DEV), torch.ones(4, device=DEV)
    r = gf.residual_norm(x, x, v, post_weight=v)
    back = gf.residual_norm_backward
    for call in (lambda: gf.linear(x, w[:, :100]), lambda: gf.linear(x, w.bfloat16()),
                 lambda: gf.linear(x.double(), w.double()), lambda: gf.linear(x, w.cpu()),
                 lambda: gf.linear(x, w, v), lambda: gf.linear(x, w, v[:7].bfloat16()),
                 lambda: gf.linear(x, w, activation="tanh"), lambda: gf.linear(x, w, residual=x),
                 lambda: gf.linear(x, w, residual=torch.ones(4, 7, device=DEV, dtype=BF16)),
                 lambda: gf.linear(x.T, w), lambda: gf.linear(v, w), lambda: gf.linear(x, None),
                 lambda: gf.linear_backward(x, w), lambda: gf.linear_backward(x[:, :7], w, x),
                 lambda: gf.linear_backward(x[:, :7], w, None, "gelu"),
                 lambda: gf.linear_backward(x[:, :7], w, x[:3], "gelu"),
                 lambda: gf.linear_backward(x[:, :7], w, residual=x[:, :100]),
                 lambda: gf.activation_backward(x, x, None), lambda: gf.activation_backward(x, None, "relu"),
                 lambda: gf.activation_backward(x, x[:, :3], "relu"), lambda: gf.activation_backward(x, x, "elu"),
                 lambda: gf.linear_weight_gradient(x, x[:3]), lambda: gf.linear_weight_gradient(x, x.bfloat16()),
                 lambda: gf.linear_weight_gradient(x, gf.checkpoint(x)),
                 lambda: gf.linear_weight_gradient(x, x, [3]),
                 lambda: gf.linear_weight_gradient(x, x, out=torch.empty(1, 200, 100, device=DEV)),
                 lambda: gf.residual_norm(x, x[:3]), lambda: gf.residual_norm(x, x.bfloat16()),
                 lambda: gf.residual_norm(x, None), lambda: gf.residual_norm(x, x, bias=v),
                 lambda: gf.residual_norm(x, x, post_bias=v), lambda: gf.residual_norm(x, x, v, v, rms=True),
                 lambda: gf.residual_norm(x, x, v, v.bfloat16()), lambda: gf.residual_norm(x, x, v[:100]),
                 lambda: gf.residual_norm(x.bfloat16(), x.bfloat16(), v, post_weight=v.bfloat16()),
                 lambda: gf.residual_norm(x, x, gate=x[:, :100]), lambda: gf.residual_norm(x, x, gate=s),
                 lambda: gf.residual_norm(x, x, gate=1.0), lambda: gf.residual_norm(x, x, y8=True),
                 lambda: gf.residual_norm(x[:, :0], x[:, :0]), lambda: back(r, x, None, None, v),
                 lambda: back(r, x, x, x), lambda: back(r, x, x, x, v, counts=[3]),
                 lambda: back(r, x, x[:3]), lambda: back(r, x, x, dweight=x),
                 lambda: back(r, x, x, x, v, dweight=x), lambda: back(r, x, x, gate=x, dgate=x[:1]),
                 lambda: back(r._replace(rstd=None), x, x, x, v), lambda: back(r._replace(s=s), x, x, x, v),
                 lambda: back(r._replace(post_mean=None), x, x, x, v, v),
                 lambda: gf.clip_gradients([], 1.0), lambda: gf.clip_gradients(x, -1.0),
                 lambda: gf.clip_gradients(x, float("nan")), lambda: gf.clip_gradients(x.double(), 1.0),
                 lambda: gf.clip_gradients(x.cpu(), 1.0), lambda: gf.clip_gradients([x, x[:3]], 1.0),
                 lambda: gf.clip_gradients(x.T, 1.0), lambda: gf.clip_gradients(v.expand(4, 200), 1.0),
                 lambda: gf.clip_gradients(x, 1.0, out=x[:, :100]), lambda: gf.gradient_norms(None),
                 lambda: gf.gradient_norms(torch.ones((), device=DEV)), lambda: gf.gradient_norms(x[:0])):
        with pytest.raises((ValueError, TypeError)):
            call()
    with pytest.raises(gf.GarfieldError):
        gf.residual_norm(x, x, v, eps=-1.0)
    with pytest.raises(gf.GarfieldError) as e:
        gf.gradient_norms(torch.ones(65, 3, device=DEV))
    assert e.value.code == gf.ETOOBIG
    assert ctypes.sizeof(worker._Gradient) == 32

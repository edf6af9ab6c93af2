"""The worker's operators at sizes that take each of their kernels' forms: every tile
of the products, tokens cut into shares, several rows of a layer norm at a time,
offsets beyond 32 bits. References are 64-bit products on the GPU; tolerances are
those of tests/test_gpu_worker.py (n terms on matrix instructions: 2 n u times the sum
of their magnitudes, u = 2^-24; then half a unit of the result's type)."""
import pytest
import torch

import paper_2010_05888_amd as gf
import worker_reference as ref
from test_gpu_worker import _dev, _gen, _norm_bound, _rand, _split
from worker_reference import BF16, F16, F32, U, close, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _library():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    gf.load()


def _values(c):
    return c.restore(F32).double()


@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(3301, 4003, 515), (1500, 2100, 700), (1409, 1999, 128),
                                   (65, 8192, 300), (4096, 3584, 257)])
def test_linear8_tiles(m, n, k, dtype, fast):
    x8 = gf.checkpoint(_rand(m, k, 1).to(DEV))
    w8 = gf.checkpoint(_rand(n, k, 2, scale=k ** -0.5).to(DEV))
    b = torch.randn(n, generator=_gen(3)).to(DEV)
    out = gf.linear8(x8, w8, b, dtype, fast)
    xv, wv = _values(x8), _values(w8)
    want = xv @ wv.T + b.double()
    size = xv.abs() @ wv.abs().T + b.double().abs()
    bound = 2 * (k + 4) * U * size + (2.0 ** -10 * size if fast else 0)
    assert bool(((out.double() - want).abs() <= bound + rounded(want.abs() + bound, dtype)).all())


@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("k", [1024, 8192, 16384, 9000])
def test_linear8_long_rows(k, fast):
    """Many groups of exponents, and checkpoints whose rows are padded by a block."""
    m, n = 130, 200
    x8 = gf.checkpoint(_rand(m, k, 1).to(DEV))
    w8 = gf.checkpoint(_rand(n, k, 2, scale=k ** -0.5).to(DEV))
    assert x8.values.stride(0) % 8192 and torch.equal(
        _values(x8), ref.blocks(_rand(m, k, 1))[0].to(DEV))
    want = _values(x8) @ _values(w8).T
    size = _values(x8).abs() @ _values(w8).abs().T
    bound = 2 * (k + 4) * U * size + (2.0 ** -10 * size if fast else 0)
    assert bool(((gf.linear8(x8, w8, dtype=F32, fast=fast).double() - want).abs() <= bound).all())


@pytest.mark.parametrize("fast", [False, True])
def test_linear8_of_rows_far_apart(fast):
    """More than 2^24 bytes between rows: offsets of 64 bits, and the same bits."""
    rows, k, apart = 70, 300, (1 << 24) + 128
    near = gf.checkpoint(_rand(rows, k, 1).to(DEV))
    w8 = gf.checkpoint(_rand(90, k, 2).to(DEV))
    flat = torch.empty(rows * apart, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    far_values = flat.as_strided((rows, 384), (apart, 1))
    far_values.copy_(near.values)
    far = gf.Checkpoint(far_values, near.exponents, k)
    assert torch.equal(gf.linear8(far, w8, fast=fast), gf.linear8(near, w8, fast=fast))
    assert torch.equal(gf.linear8(w8, far, fast=fast), gf.linear8(w8, near, fast=fast))
    few = gf.checkpoint(_rand(5, k, 3).to(DEV))
    assert torch.equal(gf.linear8(few, far), gf.linear8(few, near))


# 256 x 256 tiles, packed and not; 128 x 128; 64 x 128; tokens cut into shares
GRADIENTS = [(2, 700, 2901, 2500), (2, 700, 2904, 2433), (3, 290, 2560, 3000), (4, 300, 2000, 1000),
             (5, 900, 1001, 500), (1, 5000, 70, 130), (3, 4100, 64, 128), (2, 9000, 136, 257)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,tokens,outputs,inputs", GRADIENTS)
def test_weight_gradient_tiles(n, tokens, outputs, inputs, dtype):
    dy = _rand(tokens, outputs, 1, dtype, 0.01).to(DEV)
    x8 = gf.checkpoint(_rand(tokens, inputs, 2).to(DEV))
    counts = _split(tokens, n, outputs)
    dbias = torch.full((n, outputs), float("nan"), device=DEV)
    dw, _ = gf.weight_gradient(dy, x8, counts, dbias=dbias)
    parts = {F32: 3, F16: 2, BF16: 1}[dtype]
    for w, (d, x) in enumerate(zip(dy.double().split(counts), _values(x8).split(counts))):
        size = d.abs().T @ x.abs()
        assert bool(((dw[w].double() - d.T @ x).abs()
                     <= 2 * (parts * counts[w] + 20) * U * size + 1e-40).all())
        assert bool(((dbias[w].double() - d.sum(0)).abs()
                     <= 2 * (parts * counts[w] + 20) * U * d.abs().sum(0) + 1e-40).all())
    again, _ = gf.weight_gradient(dy, x8, counts)
    assert torch.equal(again, dw)


def test_weight_gradient_of_rows_too_far_apart():
    flat = torch.empty((1 << 26) + 4096, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    x8 = gf.Checkpoint(flat.as_strided((2, 128), ((1 << 26) + 128, 1)),
                       torch.zeros(2, 4, dtype=torch.uint8, device=DEV), 100)
    with pytest.raises(gf.GarfieldError) as e:
        gf.weight_gradient(torch.ones(2, 8, device=DEV), x8)
    assert e.value.code == gf.ETOOBIG


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["plain", "offset"])
@pytest.mark.parametrize("rows,cols", [(2051, 1031), (2049, 2500), (2050, 4096)])
def test_layernorm_of_many_rows(rows, cols, layout, dtype):
    x = _rand(rows, cols, 5, dtype)
    weight = 1 + 0.3 * torch.randn(cols, generator=_gen(1))
    bias = torch.randn(cols, generator=_gen(2))
    r = gf.layernorm(_dev(x, layout), weight.to(DEV), bias.to(DEV), 1e-5, x8=True, y8=True)
    y, mean, rstd = ref.layernorm(x, weight, bias, 1e-5)
    bound = _norm_bound(x, y, mean, rstd, weight)
    close(r.y, y, bound + rounded(y.abs() + bound, dtype), "y")
    one = gf.layernorm(_dev(x[-1:]), weight.to(DEV), bias.to(DEV), 1e-5)
    close(one.mean, r.mean[-1:].cpu().double(), 200 * U * x[-1:].double().abs().mean(1), "mean")
    x8 = gf.checkpoint(_dev(x))
    assert torch.equal(r.x8.restore(F32), x8.restore(F32))
    y8 = r.y8.restore(F32).double().cpu()
    assert float((y8 - y).abs().max() / y.abs().max()) < 2.0 ** -4


@pytest.mark.parametrize("n,rows,cols", [(19, 5000, 2500), (3, 2100, 4097), (5, 9000, 600)])
def test_layernorm_backward_of_many_rows(n, rows, cols):
    x, dy = _rand(rows, cols, 1, BF16), _rand(rows, cols, 2, BF16, 0.1)
    weight = 1 + 0.3 * torch.randn(cols, generator=_gen(4))
    _, mean, rstd = (t.float() for t in ref.layernorm(x, weight, None, 1e-5))
    counts = _split(rows, n, rows)
    dx, dw, db = gf.layernorm_backward(dy.to(DEV), gf.checkpoint(x.to(DEV)), mean.to(DEV),
                                       rstd.to(DEV), weight.to(DEV), counts)
    (rx, rw, rb), (sx, sw, sb) = ref.layernorm_backward(dy, ref.blocks(x)[0], mean, rstd, weight,
                                                        counts)
    bound = 36 * U * sx + 1e-44
    close(dx, rx, bound + rounded(rx.abs() + bound, BF16), "dx")
    close(dw, rw, (torch.tensor(counts)[:, None] + 4.0) * U * sw + 1e-44, "dweight")
    close(db, rb, (torch.tensor(counts)[:, None] + 4.0) * U * sb + 1e-44, "dbias")

"""Dense products at sizes that take each form: tiles of 256, 128, 64 and 32 lines, shares of the
depth or of the tokens, few rows, rows that are packed. Against 64-bit products on the GPU, with
test_gpu_worker_block.py's tolerances; ragged sizes, so that every tile has an edge."""
import pytest
import torch

import paper_2010_05888_amd as gf
import block_reference as ref
from test_gpu_worker import _split
from worker_reference import BF16, F16, F32, rounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [F32, BF16, F16]


def _gpu(rows, cols, seed, dtype, scale=1.0, layout="plain"):
    """Values whose columns and rows differ in size and offset; rows further apart, or one
    element into an allocation, with NaN around."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device=DEV)
    x = x * (0.2 + 3 * torch.rand(cols, generator=g, device=DEV) ** 4)
    x = ((x + 0.5 * torch.randn(cols, generator=g, device=DEV)) * scale).to(dtype)
    if layout == "plain":
        return x
    ld = cols + (8 if layout == "apart" else 5 if layout == "strided" else 0)
    flat = torch.full((rows * ld + 9,), float("nan"), dtype=dtype, device=DEV)
    at = 1 if layout == "offset" else 0
    view = flat[at:at + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(x)
    return view


def _check(got, want, dtype, what):
    value, bound = want
    over = (got.double() - value).abs() - (bound + rounded(value.abs() + bound, dtype))
    assert bool(got.isfinite().all()) and float(over.max()) <= 0, (what, float(over.max()))


# (rows, columns, depth) of: tiles of 256 (256 of them, 225), of 128 (256, 210), of 64 (uncut: 320), of 32 in
# fp32 (600), shares (80 tiles, 16, 2), few rows, a depth below a block, and one of a whole number
PRODUCTS = [(4090, 4081, 200), (2040, 2030, 330), (3700, 3650, 200), (3700, 3656, 1032), (1800, 1750, 136),
            (1795, 1750, 600), (1000, 1250, 330), (777, 1500, 1000), (300, 1000, 4096), (120, 500, 8192), (40, 100, 3000), (16, 1000, 4104),
            (15, 1003, 4100), (9, 33, 700), (300, 300, 8), (700, 640, 64)]


@pytest.mark.parametrize("layout", ["plain", "apart", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_products_of_each_form(m, n, k, dtype, layout):
    x, w = _gpu(m, k, m + k, dtype, 1.0, layout), _gpu(n, k, n, dtype, k ** -0.5, layout)
    bias, residual = torch.randn(n, device=DEV), _gpu(m, n, 5, dtype, 1.0, layout)
    name = ref.ACTIVATIONS[(m + k) % 4]
    r = gf.linear(x, w, bias, name, residual, pre=True)
    out, pre = ref.linear(x, w, bias, name, residual)
    _check(r.out, out, dtype, "out")
    _check(r.pre, pre, dtype, "pre")
    plain = gf.linear(x, w).out
    _check(plain, ref.linear(x, w, None, None, None)[0], dtype, "product")
    w2 = _gpu(k, n, n + 1, dtype, k ** -0.5, layout)
    dx = gf.linear_backward(x, w2, residual, name, residual)
    _check(dx, ref.linear_backward(x, w2, residual, name, residual), dtype, "dx")
    again = gf.linear(x, w, bias, name, residual, pre=True)
    assert torch.equal(again.out, r.out) and torch.equal(again.pre, r.pre), "other bits from another call"


# (workers, tokens, outputs, inputs): tiles of 256, 128 and 64, shares of the tokens, whole lines and not
GRADIENTS = [(16, 900, 1020, 1010), (16, 900, 500, 510), (12, 1500, 1000, 1030), (12, 1500, 1000, 1024), (19, 700, 300, 500),
             (19, 700, 320, 512), (3, 400, 130, 200), (1, 3000, 200, 300), (2, 5001, 70, 64), (60, 130, 512, 256), (1, 100, 8, 2000)]


@pytest.mark.parametrize("layout", ["plain", "apart", "strided", "offset"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,tokens,outputs,inputs", GRADIENTS)
def test_weight_gradients_of_each_form(n, tokens, outputs, inputs, dtype, layout):
    dy, x = _gpu(tokens, outputs, 1, dtype, 0.1, layout), _gpu(tokens, inputs, 2, dtype, 1.0, layout)
    counts = _split(tokens, n, n)
    dw, db = gf.linear_weight_gradient(dy, x, counts, dbias=torch.full((n, outputs), float("nan"), device=DEV))
    want = ref.weight_gradient(dy, x, counts)
    _check(dw, want[:2], F32, "dw")
    _check(db, want[2:], F32, "db")
    for w, c in enumerate(counts):
        if c == 0:
            assert not bool(dw[w].any()) and not bool(db[w].any())
    alone, _ = gf.linear_weight_gradient(dy, x, counts)
    assert torch.equal(alone, dw), "other bits without dbias"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(3700, 3650, 200), (1800, 1750, 136), (300, 1000, 4096)])
def test_large_tiles_keep_what_is_not_finite_with_its_row(m, n, k, dtype):
    x, w = _gpu(m, k, 1, dtype), _gpu(n, k, 2, dtype, k ** -0.5)
    clean = gf.linear(x, w).out
    x[m - 1, k - 1], x[5, 0] = float("nan"), float("inf")
    w2 = w.clone()
    got = gf.linear(x, w).out
    keep = [t for t in range(m) if t not in (5, m - 1)]
    assert torch.equal(got[keep], clean[keep])
    assert bool(got[m - 1].isnan().all()) and not bool(got[5].isfinite().any())
    w2[n - 1, 3] = float("nan")
    x[m - 1, k - 1] = x[5, 0] = 0
    got = gf.linear(x, w2).out
    assert bool(got[:, n - 1].isnan().all()) and bool(got[:, :n - 1].isfinite().all())


def test_rows_after_the_last_worker_are_not_read():
    """A batch padded with NaN tokens: the call sees the rows before them."""
    dy, x = _gpu(520, 300, 1, BF16), _gpu(520, 256, 2, BF16)
    want = gf.linear_weight_gradient(dy[:500].contiguous(), x[:500].contiguous(), [200, 300])[0]
    _check(want, ref.weight_gradient(dy[:500], x[:500], [200, 300])[:2], F32, "dw")
    dy[500:], x[500:] = float("nan"), float("nan")
    assert torch.equal(gf.linear_weight_gradient(dy[:500], x[:500], [200, 300])[0], want)


def test_more_inputs_than_a_product_addresses_are_refused():
    wide = torch.empty(1, (1 << 20) + 8, dtype=BF16, device=DEV)
    for call in (lambda: gf.linear(wide, wide), lambda: gf.linear_backward(wide[:, :1], wide),
                 lambda: gf.linear_weight_gradient(wide, wide[:, :8])):
        with pytest.raises(gf.GarfieldError) as e:
            call()
        assert e.value.code == gf.ETOOBIG
    x = torch.ones(17, 1 << 20, dtype=BF16, device=DEV)  # the largest
    assert gf.linear(x, x[:3]).out.tolist() == [[float(1 << 20)] * 3] * 17
    assert gf.linear_backward(x[:, :3].contiguous(), x[:3]).eq(3).all()


def test_largest_grids_of_thin_matrices():
    """Very many rows of few columns, and few rows of very many."""
    m = 1 << 22
    x = torch.ones(m, 3, dtype=BF16, device=DEV)
    assert bool(gf.linear(x, x[:5]).out.eq(3).all())
    dw, db = gf.linear_weight_gradient(x, x, [m // 2, 0, m // 2], dbias=torch.empty(3, 3, device=DEV))
    assert dw[:, 0, 0].tolist() == [m / 2, 0, m / 2] and db[:, 0].tolist() == [m / 2, 0, m / 2]
    r = gf.residual_norm(x, x, torch.ones(3, device=DEV))
    assert bool(r.s.eq(2).all()) and not bool(r.y.any())
    assert bool(gf.activation_backward(x, x, "relu").eq(1).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 16, 17, 61, 130, 5000])
@pytest.mark.parametrize("pitch,cols", [(1, 1), (1, 0), (3, 2), (5, 5), (7, 6), (8, 7), (9, 9)])
def test_matrices_that_end_with_their_memory(rows, pitch, cols, dtype):
    """Rows shorter than a block of depth (pitch and columns in 16-byte pieces, 0: three values),
    whose last one ends where a block of memory of its own does: nothing behind it is there."""
    piece = 16 // dtype.itemsize
    cols, ld = cols * piece or 3, pitch * piece

    def at_end(seed):
        memory = torch.empty((20 << 20) // dtype.itemsize, dtype=dtype, device=DEV)
        first = memory.numel() - (rows - 1) * ld - cols
        view = memory.as_strided((rows, cols), (ld, 1), first)
        view.copy_(_gpu(rows, cols, seed, dtype))
        return view

    x, w = at_end(1), at_end(2)
    _check(gf.linear(x, w).out, ref.linear(x, w, None, None, None)[0], dtype, "product")
    y = _gpu(rows, rows, 3, dtype)
    _check(gf.linear_backward(y, w), ref.linear_backward(y, w, None, None, None), dtype, "dx")
    dw, db = gf.linear_weight_gradient(x, w, dbias=torch.empty(1, cols, device=DEV))
    want = ref.weight_gradient(x, w, [rows])
    _check(dw, want[:2], F32, "dw")
    _check(db, want[2:], F32, "db")

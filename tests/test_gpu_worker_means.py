"""Layer norm of rows whose values lie close together and far from 0: the error of the mean
is an error of every value of the row."""
import pytest
import torch

import paper_2010_05888_amd as gf
import worker_reference as ref
from test_gpu_worker import _gen
from worker_reference import BF16, F16, F32, U, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# every form of the kernel: one wave, four and sixteen, two rows at a time, long rows
SIZES = [(3, 7), (5, 100), (3, 700), (4, 1500), (4, 3000), (3, 5000), (3, 9000), (2, 20000),
         (2, 40001), (2100, 1500), (2100, 3000)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    gf.load()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layernorm_of_constant_rows(rows, cols, dtype):
    """The mean of equal values is that value, so y is the bias."""
    c = torch.tensor([1234.567, -9999.9, 0.1, 3.3e-5, 777.0]).to(dtype)
    if dtype != F16:
        c[2] = -1.234e30
    c = c.repeat(rows)[:rows]
    bias = torch.randn(cols, generator=_gen(1))
    r = gf.layernorm(c[:, None].expand(rows, cols).contiguous().to(DEV), torch.ones(cols, device=DEV),
                     bias.to(DEV), 1e-5, x8=True, y8=True)
    assert torch.equal(r.mean.cpu(), c.float())
    assert torch.equal(r.y.cpu(), bias.to(dtype).expand(rows, cols))
    close(r.rstd, torch.full((rows,), 1e-5, dtype=torch.float64).rsqrt(), 8 * U * 1e-5 ** -0.5, "rstd")


@pytest.mark.parametrize("rows,cols", SIZES)
def test_layernorm_of_rows_far_from_zero(rows, cols):
    """Values that differ by 2^-9 of their offset. The differences to a mean within a few roundings
    of the true one add up, over the row, to that mean's error but for their own roundings (2^-9 u
    of the offset each, some 100 of them in a sum): the mean is off by a rounding of its own, half a
    unit each for its correction's and its own."""
    x = 5000.0 + 10.0 * torch.rand(rows, cols, generator=_gen(2))
    ones = torch.ones(cols)
    r = gf.layernorm(x.to(DEV), ones.to(DEV), None, 1e-5)
    y, mean, rstd = ref.layernorm(x, ones, None, 1e-5)
    dmean = (1 + 100 * 2.0 ** -9) * U * mean.abs()
    close(r.mean, mean, dmean, "mean")
    # y: the mean's error, and what the values in units of the deviation lose themselves
    close(r.y, y, dmean[:, None] * rstd[:, None] * 1.01 + 200 * U * y.abs(), "y")

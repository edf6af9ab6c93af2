"""The operators of a worker's residual block where a value is not finite."""
import pytest
import torch

import paper_2010_05888_amd as gf
from test_gpu_worker import _rand
from worker_reference import BF16, F16, F32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [F32, BF16, F16]

# m tokens back through k outputs to n inputs: shares of the depth, tiles of 64 lines, of 32 in fp32 and of 256
BACK = [(1, 70, 200), (40, 70, 1300), (300, 200, 96), (1800, 1750, 136)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", BACK)
def test_relu_passes_nothing_on_where_it_gave_nothing(m, n, k, dtype):
    """relu's gradient is 0 at p <= 0 whatever arrives there, infinities and NaN too."""
    dy, w, pre = _rand(m, k, 1, dtype), _rand(k, n, 2, dtype), _rand(m, n, 3, dtype)
    pre[0, :2] = 0.0
    dy[0, 3], dy[m // 2, 5] = float("inf"), float("nan")  # (m = 1: of one row)
    dy, w, pre = dy.to(DEV), w.to(DEV), pre.to(DEV)
    product = gf.linear_backward(dy, w)
    assert not bool(product[m // 2].isfinite().any())
    want = torch.where(pre > 0, product, 0.0)
    assert int((want == 0).sum()) > 0
    for got in (gf.linear_backward(dy, w, pre, "relu"), gf.activation_backward(product, pre, "relu")):
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(1.0), want.nan_to_num(1.0))
    residual = _rand(m, n, 4, dtype).to(DEV)
    got = gf.linear_backward(dy, w, pre, "relu", residual)
    assert torch.equal(got[pre <= 0], residual[pre <= 0])

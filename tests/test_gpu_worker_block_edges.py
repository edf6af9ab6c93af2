"""The operators of a worker's residual block where a value is not finite, or a slope's side decides."""
import pytest
import torch

import paper_2010_05888_amd as gf
import block_reference as ref
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


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_slopes_at_infinities(name, dtype):
    """0 far below and 1 far above, to slope_bound()."""
    inf = float("inf")
    pre = torch.tensor([[-inf, inf, -inf, inf, inf, -inf, 0.5, -0.5, inf]], dtype=dtype)
    dy = torch.tensor([[1.0, 1.0, -3.0, 0.25, -7.0, 100.0, 0.0, 0.0, 0.0]], dtype=dtype)
    got = gf.activation_backward(dy.to(DEV), pre.to(DEV), name).double().cpu()
    want = torch.where(pre > 0, dy, 0.0).double()
    off = (got - want).abs() - dy.double().abs() * ref.slope_bound(want)
    assert bool(got.isfinite().all()) and float(off.max()) <= 0


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
@pytest.mark.parametrize("m,n,k", BACK)
def test_sums_beyond_fp16_have_slopes_of_0_and_1(m, n, k, name):
    """p kept in fp16 is infinite beyond 65504; the layer's result there is p or 0, its slope 1 or 0."""
    x, w = torch.full((m, 8), 256.0, dtype=F16), torch.zeros(n, 8, dtype=F16)
    w[:, 0] = torch.where(torch.arange(n) % 3 == 0, 512.0, torch.where(torch.arange(n) % 3 == 1, -512.0, 0.001))
    up = gf.linear(x.to(DEV), w.to(DEV), None, name, pre=True)
    assert bool((up.pre[:, 0] == float("inf")).all()) and bool((up.pre[:, 1] == -float("inf")).all())
    assert bool((up.out[:, 1::3] == 0).all())
    dy, v = _rand(m, k, 1, F16, 0.1).to(DEV), _rand(k, n, 2, F16).to(DEV)
    product, got = gf.linear_backward(dy, v), gf.linear_backward(dy, v, up.pre, name)
    assert bool(got.isfinite().all())
    # a slope within slope_bound() of 1 moves the sum by a small part of an fp16 unit: the rounding's other side
    off = (got[:, ::3].double() - product[:, ::3].double()).abs() - 2.0 ** -10 * product[:, ::3].double().abs()
    assert float(off.max()) <= 2.0 ** -24
    assert float(got[:, 1::3].abs().max()) <= 2.0 ** -24  # of 0: within fp16's smallest step


@pytest.mark.parametrize("lengths", [[40], [40, 0, 90_000]])
def test_an_infinite_limit_clips_nothing(lengths):
    """Also not where a norm is infinite; a NaN is its worker's all the same."""
    grads = [_rand(4, k, 1 + k) if k else torch.empty(4, 0) for k in lengths]
    grads[0][1, 3], grads[0][1, 4], grads[0][2, 5] = float("inf"), -float("inf"), float("nan")
    here = [g.to(DEV) for g in grads]
    want = torch.cat(grads, 1)
    want[2] = float("nan")
    out = torch.empty(4, sum(lengths), device=DEV)
    norms = gf.clip_gradients(here, float("inf"), out=out)
    assert norms.isinf().tolist() == [False, True, False, False] and bool(norms[2].isnan())
    assert torch.equal(out.cpu().nan_to_num(7.0, posinf=8.0, neginf=9.0), want.nan_to_num(7.0, posinf=8.0, neginf=9.0))
    gf.clip_gradients(here, float("inf"))
    assert torch.equal(torch.cat(here, 1).cpu().nan_to_num(7.0, posinf=8.0, neginf=9.0),
                       want.nan_to_num(7.0, posinf=8.0, neginf=9.0))

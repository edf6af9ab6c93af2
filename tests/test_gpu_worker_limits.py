"""The worker's operators at widths whose launches would pass 2^32 threads."""
import pytest
import torch

import paper_2010_05888_amd as gf
from worker_reference import BF16, F32, U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _library():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    gf.load()
    yield
    torch.cuda.empty_cache()


def test_weight_gradient_of_more_tiles_than_a_launch_takes():
    """64 workers' gradients of one output and 2^25 inputs: 2^18 + 1 tiles of 128 inputs and 256
    threads each. n terms: 2 n u times the sum of their magnitudes, as on any matrix instruction."""
    n, inputs = 64, (1 << 25) + 77
    counts = [0] * n
    counts[0], counts[40], counts[62], counts[63] = 1, 2, 1, 3
    tokens = sum(counts)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x8 = gf.checkpoint(torch.randn(tokens, inputs, device=DEV, generator=gen).to(BF16))
    dy = torch.randn(tokens, 1, device=DEV, generator=gen).to(BF16)
    dbias = torch.full((n, 1), float("nan"), device=DEV)
    dw, _ = gf.weight_gradient(dy, x8, counts, dbias=dbias)
    x, at = x8.restore(F32), 0
    for w in range(n):
        d, v = dy[at:at + counts[w]].double(), x[at:at + counts[w]].double()
        at += counts[w]
        bound = 2 * (counts[w] + 4) * U * (d.abs().T @ v.abs()) + 1e-40
        assert bool(((dw[w].double() - d.T @ v).abs() <= bound).all()), w
        assert abs(float(dbias[w, 0]) - float(d.sum())) <= 2 * (counts[w] + 4) * U * float(
            d.abs().sum()) + 1e-40, w


def test_layernorm_backward_of_rows_wider_than_a_launch_of_sums():
    """2^29 + 65 columns: with a workgroup for 64 columns of dweight and dbias, their sums would take
    2^24 + 3 workgroups of 256 threads. A row's own sums: a lane adds cols / 1024 terms."""
    cols, counts = (1 << 29) + 65, [1, 0, 1]
    gen = torch.Generator(device=DEV).manual_seed(2)
    dy = torch.randn(2, cols, device=DEV, generator=gen, dtype=BF16)
    x = torch.randn(2, cols, device=DEV, generator=gen, dtype=BF16)
    mean, rstd = torch.tensor([0.25, -0.5], device=DEV), torch.tensor([1.5, 0.75], device=DEV)
    weight = torch.full((cols,), 0.5, device=DEV)
    dx, dw, db = gf.layernorm_backward(dy, x, mean, rstd, weight, counts)
    step = 1 << 26
    parts = [slice(a, min(cols, a + step)) for a in range(0, cols, step)]
    for row, worker in ((0, 0), (1, 2)):
        m, r = mean[row].double(), rstd[row].double()
        along = across = size = 0.0
        for p in parts:
            g, h = dy[row, p].double() * 0.5, (x[row, p].double() - m) * r
            along, across = along + float(g.sum()), across + float((g * h).sum())
            size += float((g * h).abs().sum() + g.abs().sum())
            want = dy[row, p].double() * h
            assert bool(((dw[worker, p].double() - want).abs() <= 8 * U * want.abs()).all())
            assert torch.equal(db[worker, p], dy[row, p].float())
        for p in parts:
            g, h = dy[row, p].double() * 0.5, (x[row, p].double() - m) * r
            want = r * (g - along / cols - h * across / cols)
            bound = r * ((cols / 1024 + 20) * U * (size / cols) * (1 + h.abs()) + 8 * U * g.abs())
            bound = bound + (want.abs() + bound) * 2.0 ** -8
            assert bool(((dx[row, p].double() - want).abs() <= bound).all())
    assert not bool(dw[1].any()) and not bool(db[1].any())

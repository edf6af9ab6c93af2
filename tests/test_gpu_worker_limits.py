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

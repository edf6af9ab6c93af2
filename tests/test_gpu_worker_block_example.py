"""The operators of a worker's residual block together, as the example trains with them:
gradients of the whole step against autograd in 64 bits, and a run with Byzantine workers."""
import math
import os
import sys

import pytest
import torch

import block_reference as ref
from test_gpu_worker import _rand

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import worker_block  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _loss(block, theta, x, dout):
    parts = theta.split([torch.Size(s).numel() for s in block.shapes.values()])
    p = {k: v.view(s) for (k, s), v in zip(block.shapes.items(), parts)}
    h = x @ p["w0"].T
    r = ref.residual_norm(x, h, p["gain"], None, p["post"], None, p["gate"], 1.0, 1e-5, True)
    up = ref.activation("gelu", r["y"][0] @ p["w1"].T + p["b1"])
    return (dout * (up @ p["w2"].T + r["s"][0])).sum()


@pytest.mark.parametrize("max_norm", [math.inf, 1e-3])
def test_gradients_of_a_step_are_the_gradients_of_its_loss(max_norm):
    """Each worker's row against autograd, in 64 bits, of sum(dout * block(x)), itself against
    differences. A dozen roundings to 16 bits on the way are off by 2^-8 of a value at most each,
    at random: 2% of a parameter's gradient in all."""
    torch.manual_seed(1)
    counts = [40, 64, 0, 56]
    block = worker_block.Block(96, 200, DEV)
    x = _rand(sum(counts), 96, 3, torch.bfloat16).to(DEV)
    dout = (torch.randn(sum(counts), 96, device=DEV) * 0.01).bfloat16()
    grads = torch.full((4, block.d), float("nan"), device=DEV)
    block.forward(x)
    norms = block.backward(dout, counts, max_norm, grads).double().cpu()
    assert not bool(grads.isnan().any())
    theta = block.theta.double().cpu()
    # the step sees the matrices in 16 bits
    at = 0
    for shape in block.shapes.values():
        size = torch.Size(shape).numel()
        if len(shape) == 2:
            theta[at:at + size] = theta[at:at + size].bfloat16().double()
        at += size
    xs, ds = x.double().cpu().split(counts), dout.double().cpu().split(counts)
    for worker in range(4):
        t = theta.clone().requires_grad_()
        if counts[worker] == 0:
            assert not bool(grads[worker].any()) and float(norms[worker]) == 0
            continue
        want = torch.autograd.grad(_loss(block, t, xs[worker], ds[worker]), t)[0]
        probe, step = torch.randn(block.d, dtype=torch.float64), 1e-5
        change = (_loss(block, theta + step * probe, xs[worker], ds[worker])
                  - _loss(block, theta - step * probe, xs[worker], ds[worker])) / (2 * step)
        assert abs(float(change - probe @ want)) <= 1e-5 * float(probe.norm() * want.norm())
        assert abs(float(norms[worker] / want.norm()) - 1) < 0.02
        got = grads[worker].double().cpu() * max(1.0, float(norms[worker]) / max_norm)
        at = 0
        for name, shape in block.shapes.items():
            size = torch.Size(shape).numel()
            part = slice(at, at + size)
            off = float((got[part] - want[part]).norm() / want[part].norm())
            assert off < 0.02, (worker, name, off)
            at += size


@pytest.mark.parametrize("rule", ["multikrum", "median"])
def test_the_example_runs(rule):
    losses = worker_block.train(rule, steps=3)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)

"""The worker's operators together, as the example trains with them: gradients of the
whole step against 64-bit ones of the same quantised step, and a run with Byzantine
workers."""
import os
import sys

import pytest
import torch

import paper_2010_05888_amd as gf
import worker_reference as ref
from test_gpu_worker import _rand

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import worker_step  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradients_of_a_step_are_the_gradients_of_its_loss():
    """Rows of the matrix of gradients against central differences, in 64 bits, of each worker's
    loss sum(dout * layer(x)). What 8 bits cost: dw sees y rounded to 4 bits (2^-4 of each factor,
    at random: 2^-4 / sqrt(tokens) of the sum, some tenths of a percent here and 3% at most); the
    norm's gradients see dout and w rounded so and x as well."""
    torch.manual_seed(1)
    counts = [40, 64, 56]
    layer = worker_step.Layer(96, 40, DEV)
    x = _rand(sum(counts), 96, 3, torch.bfloat16).to(DEV)
    dout = (torch.randn(sum(counts), 40, device=DEV) * 0.01).bfloat16()
    grads = torch.full((3, layer.d), float("nan"), device=DEV)
    layer.forward(x)
    layer.backward(dout, counts, grads)
    assert not bool(grads.isnan().any())
    theta = layer.theta.double().cpu()
    xs, ds = x.double().cpu().split(counts), dout.double().cpu().split(counts)

    def loss(worker, theta):
        gain, shift, w, b = (theta[p] for p in layer.parts)
        y = ref.layernorm(xs[worker], gain, shift, 1e-5)[0]
        return (ds[worker] * (y @ w.view(layer.shape).T + b)).sum()

    for worker in range(3):
        t = theta.clone().requires_grad_()
        want = torch.autograd.grad(loss(worker, t), t)[0]
        probe = torch.randn(layer.d, dtype=torch.float64)
        h = 1e-4
        change = (loss(worker, theta + h * probe) - loss(worker, theta - h * probe)) / (2 * h)
        assert abs(float(change - probe @ want)) <= 1e-6 * float(probe.norm() * want.norm())
        got = grads[worker].double().cpu()
        for p in layer.parts:
            off = float((got[p] - want[p]).norm() / want[p].norm())
            assert off < 0.08, (p, off)


def test_training_with_byzantine_workers():
    robust = worker_step.train("multikrum", steps=40)
    assert robust[-1] < 0.25 * robust[0]
    plain = worker_step.train("average", steps=40)
    assert not plain[-1] < plain[0]  # the reversed gradients win
    assert worker_step.train("multikrum", steps=3) == robust[:3]  # the same bits

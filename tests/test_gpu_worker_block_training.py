"""What the example with residual blocks does around its gradients: the rows that the rule takes, the
update, and the same bits from another run."""
import os
import sys

import pytest
import torch

import paper_2010_05888_amd as gf

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import worker_block  # noqa: E402

pytestmark = pytest.mark.gpu
F, N, RATE, FACTOR = 2, 11, 30.0, -10.0


@pytest.mark.parametrize("rule", ["multikrum", "median", "bulyan", "average"])
def test_a_step_takes_the_rules_aggregate_of_honest_and_reversed_rows(rule, monkeypatch):
    blocks, steps = [], []

    class Block(worker_block.Block):
        def __init__(self, *args):
            super().__init__(*args)
            blocks.append(self)

        def backward(self, dout, counts, max_norm, grads):
            norms = super().backward(dout, counts, max_norm, grads)
            assert len(counts) == N - F
            steps.append([self.theta.clone(), grads.clone(), norms, None, None, None])
            return norms

    def gar(name, grads, f, **kw):
        assert name == rule and f == F
        out = real(name, grads, f, **kw)
        steps[-1][3:] = grads.clone(), out[0].clone(), out[1]
        return out

    real = gf.gar
    monkeypatch.setattr(worker_block, "Block", Block)
    monkeypatch.setattr(worker_block.gf, "gar", gar)
    worker_block.train(rule, n=N, f=F, steps=4, rate=RATE)
    block = blocks[0]  # the other one is the teacher
    after = [s[0] for s in steps[1:]] + [block.theta]
    assert len(steps) == 4
    for (theta, honest, norms, rows, aggregate, chosen), now in zip(steps, after):
        assert rows.shape == (N, block.d) and torch.equal(rows[:N - F], honest)
        assert bool(rows.isfinite().all()) and bool(norms.isfinite().all())
        for i in range(F):
            assert torch.equal(rows[N - F + i], FACTOR * honest[i])
        # clipped rows
        assert bool((honest.double().norm(dim=1) <= 0.02 * (1 + 1e-5)).all())
        want = theta.double() - RATE * aggregate.double()
        off = 2.0 ** -24 * (want.abs() + RATE * aggregate.double().abs()) * 1.01
        assert bool(((now.double() - want).abs() <= off).all())
        if rule == "multikrum":
            # Honest rows lie within 0.04 of each other. A reversed row of norm 0.1 or more lies 0.08 from
            # each of them, so its seven nearest add up to 6 * 0.08^2 at least, theirs to 7 * 0.04^2 at most.
            assert float(norms[:F].min()) >= 0.01
            assert chosen.numel() > 0 and int(chosen.max()) < N - F


def test_another_run_gives_the_same_bits():
    assert worker_block.train("multikrum", steps=5) == worker_block.train("multikrum", steps=5)

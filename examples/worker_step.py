"""Training with Byzantine workers, from the tokens to the update, on one GPU.

n workers train a layer norm followed by a linear layer on their own batches; the
last f of them are Byzantine and send their peers' gradients reversed and amplified.
Every honest worker's gradients are computed by the worker's operators, straight
into its row of the n x d matrix that the aggregation rule takes. What the forward
pass keeps for the backward pass is kept in 8 bits.

    python examples/worker_step.py [--rule multikrum|median|bulyan|mda|average] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2010_05888_amd as gf  # noqa: E402


class Layer:
    """Layer norm, then a linear layer; parameters and gradients are columns of flat
    vectors: weight and bias of the norm, the matrix, its bias."""

    def __init__(self, inputs: int, outputs: int, device: str):
        self.shape = (outputs, inputs)
        ends = [inputs, 2 * inputs, 2 * inputs + outputs * inputs]
        self.d = ends[-1] + outputs
        self.parts = [slice(a, b) for a, b in zip([0] + ends, ends + [self.d])]
        self.theta = torch.zeros(self.d, device=device)
        self.theta[self.parts[0]] = 1
        self.theta[self.parts[2]] = torch.randn(outputs * inputs, device=device) * inputs ** -0.5

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        gain, shift, w, b = (self.theta[p] for p in self.parts)
        w = w.view(self.shape)
        self.norm = gf.layernorm(x, gain, shift, y=False, y8=True, x8=True)
        return gf.linear8(self.norm.y8, gf.checkpoint(w), b, fast=True)

    def backward(self, dout: torch.Tensor, counts, grads: torch.Tensor):
        """The gradients of the workers (counts tokens each) into the rows of grads."""
        gain, _, w, _ = (self.theta[p] for p in self.parts)
        into = [grads[:, p] for p in self.parts]
        gf.weight_gradient(dout, self.norm.y8, counts, out=into[2].view(-1, *self.shape),
                           dbias=into[3])
        w8 = gf.checkpoint(w.view(self.shape), transposed=True)
        dy = gf.linear8(gf.checkpoint(dout), w8, fast=True)
        return gf.layernorm_backward(dy, self.norm.x8, self.norm.mean, self.norm.rstd,
                                     gain, counts, dweight=into[0], dbias=into[1])[0]


def train(rule: str = "multikrum", n: int = 11, f: int = 2, steps: int = 60, inputs: int = 256,
          outputs: int = 130, tokens: int = 96, rate: float = 30.0, seed: int = 0):
    """The honest workers' loss before every step."""
    torch.manual_seed(seed)
    device, honest = "cuda", n - f
    layer = Layer(inputs, outputs, device)
    teacher = torch.randn(inputs, outputs, device=device) * inputs ** -0.5
    counts = [tokens + 3 * i for i in range(honest)]  # unequal batches
    share = torch.tensor(counts, device=device).reciprocal().repeat_interleave(
        torch.tensor(counts, device=device))[:, None]
    grads = torch.zeros(n, layer.d, device=device)
    losses = []
    for _ in range(steps):
        x = torch.randn(sum(counts), inputs, device=device).bfloat16()
        error = layer.forward(x).float() - x.float() @ teacher
        losses.append(float((error.square() * share).sum() / (2 * outputs * honest)))
        layer.backward((error * share / outputs).bfloat16(), counts, grads[:honest])
        gf.attack("reverse", grads[:honest], f, -10.0, out=grads[honest:])
        layer.theta -= rate * gf.gar(rule, grads, f)[0]
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rule", default="multikrum")
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    losses = train(a.rule, steps=a.steps)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i:4d}  loss {losses[i]:.4f}")
    print(f"{a.rule}: loss {losses[0]:.4f} -> {losses[-1]:.4f}")


if __name__ == "__main__":
    main()

"""Training residual blocks with Byzantine workers, in 16 bits, on one GPU.

n workers train a residual block (a linear layer, normed, gated and added to its input, then a
normed two-layer network added to that) on their own batches; the last f of them are Byzantine
and send their peers' gradients reversed and amplified. Every honest worker's gradient is
computed by the worker's operators, clipped by its norm over all the block's tensors on its way
into its row of the n x d matrix that the aggregation rule takes.

    python examples/worker_block.py [--rule multikrum|median|bulyan|mda|average] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2010_05888_amd as gf  # noqa: E402


class Block:
    """s = x + gate * N(x w0^T), out = s + gelu(N(s) w1^T + b1) w2^T, with N norms by the root
    mean square; the parameters are columns of one flat vector, in the order of `shapes`."""

    def __init__(self, width: int, hidden: int, device: str):
        self.shapes = {"w0": (width, width), "post": (width,), "gate": (width,), "gain": (width,),
                       "w1": (hidden, width), "b1": (hidden,), "w2": (width, hidden)}
        self.d = sum(torch.Size(s).numel() for s in self.shapes.values())
        self.theta = torch.empty(self.d, device=device)
        for name, p in self.parameters().items():
            if len(p.shape) == 2:
                p.copy_(torch.randn(p.shape, device=device) * p.shape[1] ** -0.5)
            else:
                p.fill_({"post": 1.0, "gate": 0.5, "gain": 1.0, "b1": 0.0}[name])

    def parameters(self):
        parts = self.theta.split([torch.Size(s).numel() for s in self.shapes.values()])
        return {name: part.view(shape) for (name, shape), part in zip(self.shapes.items(), parts)}

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        p = self.parameters()
        self.x = x
        self.w0, self.w1, self.w2 = (p[k].to(x.dtype) for k in ("w0", "w1", "w2"))
        self.h = gf.linear(x, self.w0).out
        self.r = gf.residual_norm(x, self.h, p["gain"], post_weight=p["post"], gate=p["gate"],
                                  rms=True)
        self.up = gf.linear(self.r.y, self.w1, p["b1"], "gelu", pre=True)
        return gf.linear(self.up.out, self.w2, residual=self.r.s).out

    def backward(self, dout: torch.Tensor, counts, max_norm: float, grads: torch.Tensor):
        """The workers' gradients (counts tokens each), clipped, into the rows of grads: their
        norms before."""
        p, n = self.parameters(), len(counts)
        dw2, _ = gf.linear_weight_gradient(dout, self.up.out, counts)
        dp = gf.linear_backward(dout, self.w2, self.up.pre, "gelu")
        db1 = torch.empty(n, *self.shapes["b1"], device=grads.device)
        dw1, _ = gf.linear_weight_gradient(dp, self.r.y, counts, dbias=db1)
        dy = gf.linear_backward(dp, self.w1)
        b = gf.residual_norm_backward(self.r, self.h, dout, dy, p["gain"], p["post"],
                                      gate=p["gate"], rms=True, counts=counts)
        dw0, _ = gf.linear_weight_gradient(b.dh, self.x, counts)
        return gf.clip_gradients([dw0, b.dpost_weight, b.dgate, b.dweight, dw1, db1, dw2], max_norm,
                                 out=grads)


def train(rule: str = "multikrum", n: int = 11, f: int = 2, steps: int = 60, width: int = 128,
          hidden: int = 320, tokens: int = 96, rate: float = 30.0, max_norm: float = 0.02,
          seed: int = 0):
    """The honest workers' loss before every step."""
    torch.manual_seed(seed)
    device, honest = "cuda", n - f
    block, teacher = Block(width, hidden, device), Block(width, hidden, device)
    counts = [tokens + 3 * i for i in range(honest)]  # unequal batches
    share = torch.tensor(counts, device=device).reciprocal().repeat_interleave(
        torch.tensor(counts, device=device))[:, None]
    grads = torch.zeros(n, block.d, device=device)
    losses = []
    for _ in range(steps):
        x = torch.randn(sum(counts), width, device=device).bfloat16()
        error = block.forward(x).float() - teacher.forward(x).float()
        losses.append(float((error.square() * share).sum() / (2 * width * honest)))
        block.backward((error * share / width).bfloat16(), counts, max_norm, grads[:honest])
        gf.attack("reverse", grads[:honest], f, -10.0, out=grads[honest:])
        block.theta -= rate * gf.gar(rule, grads, f)[0]
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

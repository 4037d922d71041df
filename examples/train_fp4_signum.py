"""Signum with majority vote on gradients made by 4-bit products, clipped on the way, then the trained weights served in 4 bits.

Every worker runs the same two-layer perceptron on its own mini-batches of a synthetic regression task:

    fp4.linear_forward / linear_backward   the layers' products in 4 bits; weight gradients, one tensor a layer
    binding.tensors_clip                   norm over all tensors of a worker, clipping, into the worker's row [M][ld]
    binding.signsgd_step                   momentum, signs, vote and update of the flat parameter vector (Algorithms 2, 3)

The parameters are one flat float32 vector, as the step wants it; a layer's weight is a view of it.

    python examples/train_fp4_signum.py [--steps 60] [--workers 4] [--fmt mx|nv]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1802_04434_b200 import binding as B, fp4  # noqa: E402


def up(n, k):
    return (n + k - 1) // k * k


class Perceptron:
    """x -> relu(x w1^T) w2^T with its weights in one flat vector; gradients go to tensors given by the caller."""

    def __init__(self, sides, flat, fmt):
        self.fmt, self.weights, at = fmt, [], 0
        for n_in, n_out in zip(sides, sides[1:]):
            self.weights.append(flat[at:at + n_in * n_out].view(n_out, n_in))
            at += up(n_in * n_out, 32)

    def loss_and_gradients(self, x, target, grads):
        y, kept = x, []
        for i, w in enumerate(self.weights):
            z, k = fp4.linear_forward(y, w, self.fmt)
            kept.append((k, z))
            y = torch.relu(z) if i + 1 < len(self.weights) else z
        off = y.float() - target
        dy = (off * (2.0 / off.numel())).to(x.dtype)
        for i in reversed(range(len(self.weights))):
            k, z = kept[i]
            if i + 1 < len(self.weights):
                dy = dy * (z > 0)
            dy, _ = fp4.linear_backward(k, dy, dw=grads[i])
        return off.square().mean()


def train(steps=60, workers=4, fmt="mx", batch=256, sides=(64, 256, 32), beta=0.9, delta=1e-3, max_norm=0.05, seed=0, device="cuda"):
    """Losses of the steps (mean over the workers), norms of the last step, and the trained flat vector."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    sizes = [a * b for a, b in zip(sides, sides[1:])]
    d = sum(up(n, 32) for n in sizes)
    x = torch.zeros(d, device=device)                       # parameters; what lies between the tensors stays out of the model
    net = Perceptron(sides, x, fmt)
    for w in net.weights:
        w.copy_(torch.randn(w.shape, generator=g, device=device) / w.shape[1] ** 0.5)
    task = torch.randn(sides[-1], sides[0], generator=g, device=device) / sides[0] ** 0.5

    rows = torch.zeros(workers, d, device=device)           # the step's g: one row a worker
    m = torch.zeros(workers, d, device=device)
    words = up((d + 31) // 32, 4)
    bits = torch.zeros(workers, words, dtype=torch.int32, device=device)
    vote = torch.zeros((d + 31) // 32, dtype=torch.int32, device=device)
    grads = [[torch.zeros_like(w) for w in net.weights] for _ in range(workers)]
    slices = [p[:n].view_as(w) for row in rows for p, n, w in zip(row.split([up(n, 32) for n in sizes]), sizes, net.weights)]
    table = B.TensorTable([t for per in grads for t in per], slices, [w for w in range(workers) for _ in sizes])
    norms = torch.zeros(workers, device=device)

    losses = []
    for _ in range(steps):
        loss = 0.0
        for w in range(workers):
            inputs = torch.randn(batch, sides[0], generator=g, device=device)
            target = torch.relu(inputs @ task.t())
            loss = loss + net.loss_and_gradients(inputs.bfloat16(), target, grads[w])
        B.tensors_clip(table, max_norm, norms, zero_nonfinite=True)
        B.signsgd_step(x, rows, m, workers, d, d, beta, delta, bits, words, vote)
        losses.append(loss / workers)
    fp4.check()
    return torch.stack(losses).tolist(), norms.tolist(), net, task


def serve(net, task, tokens=1, seed=1):
    """Relative error of the trained network on single inputs, its weights packed once."""
    packed = [fp4.quantise(w, net.fmt) for w in net.weights]
    g = torch.Generator(device=task.device)
    g.manual_seed(seed)
    worst = 0.0
    for _ in range(16):
        x = torch.randn(tokens, task.shape[1], generator=g, device=task.device)
        y = x.bfloat16()
        for i, w in enumerate(packed):
            y = fp4.matmul(fp4.quantise(y, net.fmt), w, torch.bfloat16)
            y = torch.relu(y) if i + 1 < len(packed) else y
        want = torch.relu(x @ task.t())
        worst = max(worst, float((y.float() - want).norm() / want.norm()))
    return worst


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--workers", type=int, default=4)
    p.add_argument("--fmt", choices=("mx", "nv"), default="mx")
    a = p.parse_args()
    losses, norms, net, task = train(a.steps, a.workers, a.fmt)
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.4f" % (k, losses[k]))
    print("step %4d  loss %.4f  gradient norms %s" % (a.steps - 1, losses[-1], ["%.3g" % n for n in norms]))
    print("single inputs through the packed weights: relative error at most %.3f" % serve(net, task))


if __name__ == "__main__":
    main()

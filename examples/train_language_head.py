"""A small next-token model with a large vocabulary, trained on both ends of what this package offers around the signSGD step:

    fp4.linear                       the hidden layers' products in 4 bits, for torch's autograd
    loss.cross_entropy               the loss over the vocabulary, its logits never in memory, with both gradients
    binding.tensors_clip             one norm over all gradients, clipping, into the step's row and in place
    orthogonal.momentum_step         hidden matrices, a batch of one shape in one call: updates with singular values near one
    binding.signsgd_step             embedding and head: momentum, signs, update (Algorithm 2, one worker)

Tokens follow a random permutation with some noise, so that the next one can be learnt from the last; a part of each batch is padding.

    python examples/train_language_head.py [--steps 60] [--vocab 2000]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1802_04434_b200 import binding as B, fp4, loss, orthogonal  # noqa: E402

PADDING = -100


def up(n, k):
    return (n + k - 1) // k * k


class Model:
    """embedding -> blocks of relu(x w^T) added to x -> head; parameters are views of one flat float32 vector: embedding, head, then the
    blocks' matrices side by side."""

    def __init__(self, vocab, width, blocks, fmt, gen, device):
        self.vocab, self.width, self.blocks, self.fmt = vocab, width, blocks, fmt
        table = up(vocab * width, 32)
        self.signs = 2 * table                                # of the flat vector: what the signs move
        self.flat = torch.zeros(self.signs + blocks * width * width, device=device)
        self.embedding = self.flat[:vocab * width].view(vocab, width)
        self.head = self.flat[table:table + vocab * width].view(vocab, width)
        self.hidden = self.flat[self.signs:].view(blocks, width, width)
        for p, size in ((self.embedding, 1.0), (self.head, 0.02), (self.hidden, width ** -0.5)):
            p.copy_(torch.randn(p.shape, generator=gen, device=device) * size)

    def parameters(self):
        """What gradients are wanted of, as torch sees it: 16-bit tables, as the loss takes them, and the blocks' matrices."""
        return [p.detach().requires_grad_() for p in (self.embedding.bfloat16(), self.head.bfloat16(), *self.hidden)]

    def loss(self, parameters, tokens, targets):
        embedding, head, *hidden = parameters
        x = torch.nn.functional.embedding(tokens, embedding)
        for w in hidden:
            x = x + torch.relu(fp4.linear(x, w, self.fmt))
        return loss.cross_entropy(x, head, targets, ignore_index=PADDING)


def batch(gen, permutation, size, device):
    vocab = permutation.numel()
    tokens = torch.randint(0, vocab, (size,), generator=gen, device=device)
    targets = permutation[tokens]
    noise = torch.rand(size, generator=gen, device=device)
    targets = torch.where(noise < 0.05, torch.randint(0, vocab, (size,), generator=gen, device=device), targets)
    return tokens, torch.where(noise > 0.9, PADDING, targets)


def train(steps=60, vocab=2000, width=128, blocks=3, size=1024, fmt="mx", beta=0.9, delta_signs=2e-3, delta_hidden=0.02, max_norm=1.0, seed=0, device="cuda"):
    """Losses and gradient norms of the steps, and the model."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    model = Model(vocab, width, blocks, fmt, gen, device)
    permutation = torch.randperm(vocab, generator=gen, device=device)
    momentum = torch.zeros_like(model.flat)
    row = torch.zeros_like(model.flat)                        # the clipped gradient, laid out as the parameters
    d = model.signs
    words = up(d // 32, 4)
    bits, vote = torch.zeros(words, dtype=torch.int32, device=device), torch.zeros(d // 32, dtype=torch.int32, device=device)
    table_size = up(vocab * width, 32)
    grads = [torch.zeros(vocab, width, dtype=torch.bfloat16, device=device) for _ in range(2)] + [torch.zeros(width, width, device=device) for _ in range(blocks)]
    places = [row[:vocab * width], row[table_size:table_size + vocab * width], *row[d:].view(blocks, width, width)]
    table = B.TensorTable(grads, [p.view_as(g) for p, g in zip(places, grads)])
    norm = torch.zeros(1, device=device)
    losses, norms = [], []
    for _ in range(steps):
        tokens, targets = batch(gen, permutation, size, device)
        parameters = model.parameters()
        value = model.loss(parameters, tokens, targets)
        for g, new in zip(grads, torch.autograd.grad(value, parameters)):
            g.copy_(new)
        B.tensors_clip(table, max_norm, norm, zero_nonfinite=True)
        B.signsgd_step(model.flat[:d], row[:d], momentum[:d], 1, d, d, beta, delta_signs, bits, words, vote)
        hidden = [t[d:].view(blocks, width, width) for t in (model.flat, row, momentum)]
        orthogonal.momentum_step(*hidden, beta, delta_hidden, nesterov=True)
        losses.append(value.detach())
        norms.append(norm.clone())
    fp4.check()
    loss.check()
    return torch.stack(losses).tolist(), torch.cat(norms).tolist(), model


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--vocab", type=int, default=2000)
    p.add_argument("--fmt", choices=("mx", "nv"), default="mx")
    a = p.parse_args()
    losses, norms, _ = train(a.steps, a.vocab, fmt=a.fmt)
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d  loss %.4f  gradient norm %.3g" % (k, losses[k], norms[k]))
    print("step %4d  loss %.4f  gradient norm %.3g" % (a.steps - 1, losses[-1], norms[-1]))


if __name__ == "__main__":
    main()

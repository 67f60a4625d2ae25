"""Weighted parallel SGD of a linear model with many classes: a language model's output layer with a head for each of the next few tokens.

    python examples/many_class_workers.py

k workers of unequal speed train the heads from the same start, each on mini-batches of its own sample stream, with gradients clipped over all
heads together; the models are averaged with the weights of Eq. 6 and answer by drawing classes.  The products run in 8-bit floating
point; weights and gradients are kept in fp32.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1708_04801_amd import api  # noqa: E402


def data_set(m, d, classes, heads, seed=0):
    """rows of normal values in bfloat16, and for each head the class that a hidden layer scores highest on them, noise added"""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(m, d, generator=gen, device="cuda").to(torch.bfloat16)
    labels = []
    for _ in range(heads):
        hidden = torch.randn(classes, d, generator=gen, device="cuda")
        noise = torch.randn(m, classes, generator=gen, device="cuda")
        labels.append((x.float() @ hidden.t() + 0.5 * d ** 0.5 * noise).argmax(1))
    return x, labels


class Heads:
    """The class vectors of all heads, in one row of the workers' models, with their gradients."""

    def __init__(self, row, classes, d, heads):
        self.weights = list(row.view(heads, classes, d).unbind(0))
        self.grads = [torch.empty_like(w) for w in self.weights]
        self.tensors = api.wpsgd_tensor_list(self.grads, self.weights)

    def scores(self, rows8):
        """of a batch, for each head"""
        for w in self.weights:
            w8 = api.wpsgd_quantize(api.Matrix(w.shape[0], w.shape[1], dense=w))
            yield api.wpsgd_block_matmul(rows8, w8)

    def step(self, X, labels, rows, eta, lam, max_norm):
        """one clipped step on a batch; the batch's mean loss over all heads, on the GPU"""
        n = rows.numel()
        rows8, columns8 = api.wpsgd_quantize(X, rows=rows), api.wpsgd_quantize(X, rows=rows, transpose=True)
        total = 0.0
        for z, y, g in zip(self.scores(rows8), labels, self.grads):
            loss, dz = api.wpsgd_softmax_loss(z, y[rows], scale=1.0 / n, grad=z)
            dz8 = api.wpsgd_quantize(api.Matrix(n, dz.shape[1], dense=dz), transpose=True)
            api.wpsgd_block_matmul(dz8, columns8, out=g)
            total = total + loss.mean()
        api.wpsgd_clipped_step(self.tensors, eta, lam, max_norm)
        return total / len(self.weights)

    def loss(self, X, labels):
        rows8 = api.wpsgd_quantize(X)
        losses = [api.wpsgd_softmax_loss(z, y, grad=False)[0].mean() for z, y in zip(self.scores(rows8), labels)]
        return float(sum(losses) / len(losses))

    def answer(self, X, u, **rule):
        """a class for each row and head"""
        rows8 = api.wpsgd_quantize(X)
        return torch.stack([api.wpsgd_draw_classes(z, u, **rule)[0] for z in self.scores(rows8)], 1)


def train(m=16384, d=512, classes=1000, heads=2, steps=(400, 400, 300, 150), batch=512, eta=4.0, lam=1e-4, max_norm=0.5, seed=7):
    """Returns the held-out losses of the start, of each worker and of the weighted average, and the average's drawn answers with the labels."""
    x, labels = data_set(m + 2048, d, classes, heads)
    X, held = api.Matrix(m, d, dense=x[:m]), api.Matrix(2048, d, dense=x[m:])
    held_labels = [y[m:].contiguous() for y in labels]
    W = torch.zeros(len(steps), heads * classes * d, device="cuda")
    start = Heads(W[0], classes, d, heads).loss(held, held_labels)
    losses = []
    for k, n in enumerate(steps):
        worker = Heads(W[k], classes, d, heads)
        for step in range(n):
            rows = api.wpsgd_sample_indices_device(seed, k, step * batch, batch, m)
            worker.step(X, labels, rows, eta, lam, max_norm)
        losses.append(worker.loss(held, held_labels))
    average = api.wpsgd_combine(W, api.wpsgd_weights(list(steps), eta, lam))
    model = Heads(average, classes, d, heads)
    u = torch.rand(2048, generator=torch.Generator().manual_seed(seed)).cuda()
    answers = model.answer(held, u, temperature=0.7, top_k=50, top_p=0.95)
    return start, losses, model.loss(held, held_labels), answers, torch.stack(held_labels, 1)


if __name__ == "__main__":
    start, workers, average, answers, labels = train()
    print(f"held-out loss: start {start:.3f}, workers {', '.join(f'{v:.3f}' for v in workers)}, weighted average {average:.3f}")
    print(f"drawn answers that are the label: {float((answers == labels).float().mean()):.3f} (by chance 0.001)")

"""Weighted parallel SGD of a linear model with many classes: a language model's output layer with a head for each of the next few tokens.

    python examples/many_class_workers.py

k workers of unequal speed train the heads from the same start, each on mini-batches of its own sample stream, with gradients clipped over all
heads together; the models are averaged with the weights of Eq. 6 and answer by drawing classes.  The products run in 8-bit floating
point; weights and gradients are kept in fp32.  A worker's heads are then tuned on the answers that they draw (those that are right are
rewarded, and they are held to what they were) and on pairs of a right and a drawn answer, with elements of the rows dropped, and served with class vectors of four bits.
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

    def _descend(self, gradients, columns8, eta, lam, max_norm):
        """one clipped step, given the gradients of all heads' scores"""
        for dz, g in zip(gradients, self.grads):
            dz8 = api.wpsgd_quantize(api.Matrix(dz.shape[0], dz.shape[1], dense=dz), transpose=True)
            api.wpsgd_block_matmul(dz8, columns8, out=g)
        api.wpsgd_clipped_step(self.tensors, eta, lam, max_norm)

    def _dropped(self, X, rows, drop, seed, chain, step):
        """a batch with elements dropped, as rows and as columns"""
        x = api.wpsgd_dropout(X, drop, seed, chain=chain, step=step, rows=rows)
        D = api.Matrix(rows.numel(), X.d, dense=x)
        return api.wpsgd_quantize(D), api.wpsgd_quantize(D, transpose=True)

    def reward_step(self, before, X, labels, rows, u, drop, seed, step, eta, lam, max_norm, kl=0.02):
        """One step on answers drawn for a batch: a right one is worth 1, compared with the batch's mean; `before` are the heads that the answers shall not
        stray far from.  Returns the share of right answers."""
        rows8, columns8 = self._dropped(X, rows, drop, seed, 0, step)
        gradients, right = [], 0.0
        for z, z0, y in zip(self.scores(rows8), before.scores(rows8), labels):
            drawn, _ = api.wpsgd_draw_classes(z, u)
            reward = (drawn == y[rows]).float()
            reference = -api.wpsgd_softmax_loss(z0, drawn, grad=False)[0]
            _, _, dz = api.wpsgd_policy_loss(z, drawn, reward - reward.mean(), ref_log=reference, kl=kl, scale=1.0 / rows.numel(), grad=z)
            gradients.append(dz)
            right = right + reward.mean()
        self._descend(gradients, columns8, eta, lam, max_norm)
        return right / len(labels)

    def preference_step(self, before, X, labels, rows, u, drop, seed, step, eta, lam, max_norm, beta=1.0):
        """One step on pairs, a row's label before an answer drawn for it.  Returns the mean margin."""
        twice = rows.repeat_interleave(2)
        rows8, columns8 = self._dropped(X, twice, drop, seed, 1, step)
        ends = torch.arange(twice.numel() + 1, device="cuda")
        gradients, margins = [], 0.0
        for z, z0, y in zip(self.scores(rows8), before.scores(rows8), labels):
            answers, _ = api.wpsgd_draw_classes(z0, u.repeat_interleave(2))
            answers[0::2] = y[rows]
            reference = -api.wpsgd_softmax_loss(z0, answers, grad=False)[0]
            _, margin, dz = api.wpsgd_preference_loss(z, answers, ends, ref_log=reference, beta=beta, scale=1.0 / rows.numel(), grad=z)
            gradients.append(dz)
            margins = margins + margin.mean()
        self._descend(gradients, columns8, eta, lam, max_norm)
        return margins / len(labels)

    def four_bits(self, group=64):
        """the class vectors as they are served"""
        return [api.wpsgd_quantize_nibbles(api.Matrix(w.shape[0], w.shape[1], dense=w), group=group) for w in self.weights]

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


def tune(row, X, labels, classes, d, heads, steps=50, batch=512, eta=1.0, lam=1e-4, max_norm=0.5, drop=0.1, seed=11):
    """Trains heads (one row of weights, changed in place) on rewarded answers and on pairs.  Returns the share of right answers before and after each step, and the margins of the pairs."""
    model, before = Heads(row, classes, d, heads), Heads(row.clone(), classes, d, heads)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    right, margins = [], []
    for step in range(steps):
        rows = api.wpsgd_sample_indices_device(seed, 0, step * batch, batch, X.m)
        u = torch.rand(batch, generator=gen, device="cuda")
        right.append(model.reward_step(before, X, labels, rows, u, drop, seed, step, eta, lam, max_norm))
        margins.append(model.preference_step(before, X, labels, rows, u, drop, seed, step, eta, lam, max_norm))
    return torch.stack(right), torch.stack(margins)


def serve(vectors, X, rows, u, **rule):
    """a class for each picked row and head, from class vectors of four bits"""
    return torch.stack([api.wpsgd_draw_classes(api.wpsgd_nibble_matmul(X, w, rows=rows), u, **rule)[0] for w in vectors], 1)


def main(m=16384, d=512, classes=1000, heads=2):
    start, workers, average, answers, labels = train(m=m, d=d, classes=classes, heads=heads)
    print(f"held-out loss: start {start:.3f}, workers {', '.join(f'{v:.3f}' for v in workers)}, weighted average {average:.3f}")
    print(f"drawn answers that are the label: {float((answers == labels).float().mean()):.3f} (by chance 0.001)")
    x, y = data_set(m, d, classes, heads, seed=1)
    X = api.Matrix(m, d, dense=x)
    row = torch.zeros(heads * classes * d, device="cuda")
    worker = Heads(row, classes, d, heads)
    for step in range(100):
        worker.step(X, y, api.wpsgd_sample_indices_device(1, 0, step * 512, 512, m), 4.0, 1e-4, 0.5)
    right, margins = tune(row, X, y, classes, d, heads)
    print(f"tuned on its answers: right {float(right[0]):.3f} -> {float(right[-1]):.3f}, margins {float(margins[0]):.3f} -> {float(margins[-1]):.3f}")
    rows, u = torch.arange(16, device="cuda"), torch.rand(16, device="cuda")
    served = serve(worker.four_bits(), X, rows, u, temperature=0.7, top_k=50)
    print(f"sixteen rows served in four bits: {int((served == torch.stack(y, 1)[:16]).sum())} of {served.numel()} answers are the label")


if __name__ == "__main__":
    main()

"""Local training of N workers on one GPU, round by round: every worker steps on its own samples, then the
synchronization round mixes the models (segmented gossip).

All workers' parameters are one flat [N][P] array, their gradients another; every layer is a view into it.  One
round is

    products grouped by worker -> group norm with SiLU -> dropout                forward
    combo_grouped_cross_entropy   the classifier and its loss, the logits never kept
    the same backwards, gradients written into the flat gradient array
    combo_grad_clip            every worker's gradient clipped by its norm over all its tensors
    combo_segment_aggregate_sgd  the SGD step and the segment-wise aggregation with R peers in one pass

    python examples/local_step.py [--workers 8] [--rounds 30] [--dtype bf16] [--dropout 0.1]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1908_07782_b200 as combo  # noqa: E402


class Workers:
    """N copies of a two-layer classifier (n_in -> width, group norm, SiLU, width -> classes), each on its own samples."""

    def __init__(self, counts, n_in, width, classes, groups, dtype=torch.float32, device="cuda", seed=0,
                 dropout=0.0):
        self.N, self.n_in, self.width, self.classes, self.groups = len(counts), n_in, width, classes, groups
        self.dtype, self.device, self.dropout, self.seed = dtype, torch.device(device), dropout, seed
        shapes = {"w1": (width, n_in), "gamma": (width,), "beta": (width,), "w2": (classes, width)}
        self.places, at = {}, 0
        for name, shape in shapes.items():
            n = 1
            for s in shape:
                n *= s
            self.places[name] = (at, n, shape)
            at += (n + 7) // 8 * 8                 # layers on 16-byte boundaries, in either type
        self.P = at
        g = torch.Generator(device="cpu").manual_seed(seed)
        start = torch.zeros(self.P)
        start[self.places["w1"][0]:][:width * n_in] = torch.randn(width * n_in, generator=g) / n_in ** 0.5
        start[self.places["gamma"][0]:][:width] = 1.0
        start[self.places["w2"][0]:][:classes * width] = torch.randn(classes * width, generator=g) / width ** 0.5
        self.params = start.repeat(self.N, 1).to(self.device)      # all workers start from one model
        self.next = torch.empty_like(self.params)
        self.grads, self.clipped = torch.zeros_like(self.params), torch.zeros_like(self.params)
        self.begin = torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int64, device=self.device)
        self.sizes = torch.tensor(counts, dtype=torch.float32, device=self.device)
        M = self.M = sum(counts)

        def rows(n, t=dtype):
            return torch.empty(M, n, dtype=t, device=self.device)

        self.h, self.a, self.da, self.dh = rows(width), rows(width), rows(width), rows(width)
        self.loss, self.lse = torch.empty(M, device=self.device), torch.empty(M, device=self.device)
        self.mean, self.rstd = rows(groups, torch.float32), rows(groups, torch.float32)
        self.scratch = torch.empty(combo.combo_group_norm_scratch_bytes(M, 1, width, groups), dtype=torch.uint8,
                                   device=self.device)
        size = 4 if dtype == torch.float32 else 2
        need = max(combo.combo_grouped_cross_entropy_scratch_bytes(self.N, M, width, classes, size, grad) for grad in (0, 4))
        self.loss_scratch = torch.empty(need, dtype=torch.uint8, device=self.device)
        # one entry for each layer of each worker; both arrays keep their places from step to step
        offsets = torch.tensor([w * self.P + a for w in range(self.N) for a, _, _ in self.places.values()]) * 4
        lengths = [n for _ in range(self.N) for _, n, _ in self.places.values()]
        self.tensors = (self.grads.data_ptr() + offsets).to(self.device)
        self.outs = (self.clipped.data_ptr() + offsets).to(self.device)
        self.starts = torch.tensor([0] + list(torch.tensor(lengths).cumsum(0)), dtype=torch.int64, device=self.device)
        self.first = torch.arange(self.N + 1, dtype=torch.int32, device=self.device) * len(self.places)
        self.total = sum(lengths)
        self.norm, self.coef = torch.empty(self.N, device=self.device), torch.empty(self.N, device=self.device)
        self.clip_scratch = torch.empty(combo.combo_grad_scratch_bytes(self.N), dtype=torch.uint8, device=self.device)

    def view(self, flat, name):
        """A layer of every worker: [N, ...] inside a flat [N][P] array."""
        at, n, shape = self.places[name]
        part = flat[:, at:at + n]
        return part if len(shape) == 1 else part.unflatten(1, shape)

    def drop(self, t, rnd):
        """Dropout in place: of the activations, and, with the same mask, of their gradient."""
        if self.dropout:
            combo.combo_dropout(t, None, t, self.begin, self.dropout, self.seed, rnd)

    def forward(self, x, flat, rnd=0):
        """What the classifier sees of every sample."""
        one = lambda t: t.view(self.M, 1, self.width)  # noqa: E731  a sample is one position
        combo.combo_grouped_linear(x, self.view(flat, "w1"), self.h, self.begin)
        combo.combo_group_norm(one(self.h), one(self.a), self.view(flat, "gamma"), self.view(flat, "beta"), self.begin,
                               self.groups, 1e-5, combo.ACT_SILU, self.mean, self.rstd, self.scratch)
        self.drop(self.a, rnd)
        return self.a

    def backward(self, x, labels, flat, rnd=0):
        """Every sample's loss, and gradients of every worker's mean into the flat gradient array."""
        one = lambda t: t.view(self.M, 1, self.width)  # noqa: E731
        w2 = self.view(flat, "w2")
        combo.combo_grouped_cross_entropy(self.a, w2, labels, self.loss, self.lse, self.begin, self.loss_scratch)
        combo.combo_grouped_cross_entropy_backward(self.a, w2, labels, self.lse, None, self.da, self.view(self.grads, "w2"), self.begin,
                                                   self.loss_scratch)
        self.drop(self.da, rnd)
        combo.combo_group_norm_backward(one(self.da), one(self.h), one(self.dh), self.view(flat, "gamma"), self.view(flat, "beta"),
                                        self.begin, self.groups, combo.ACT_SILU, self.mean, self.rstd,
                                        self.view(self.grads, "gamma"), self.view(self.grads, "beta"), self.scratch)
        combo.combo_grouped_linear_grad_weight(self.dh, x, self.view(self.grads, "w1"), self.begin)
        return self.loss

    def step(self, x, labels, lr, max_norm, rnd, segments, replicas, seed=1):
        """One round: local step of every worker, then the gossip round.  Returns the loss over all samples."""
        flat = self.params if self.dtype == torch.float32 else self.params.to(self.dtype)
        self.forward(x, flat, rnd)
        loss = self.backward(x, labels, flat, rnd).mean()
        combo.combo_grad_clip(self.tensors, self.outs, self.starts, self.first, len(self.tensors), self.N, self.total, 4,
                              max_norm, self.norm, self.coef, self.clip_scratch)
        idx = torch.empty((self.N, segments, replicas), dtype=torch.int32, device=self.device)
        combo.combo_select_peers(seed, rnd, self.N, segments, replicas, idx)
        combo.combo_segment_aggregate_sgd(self.params, self.clipped, lr, self.next, self.sizes, idx, self.N, self.P, segments,
                                          replicas)
        self.params, self.next = self.next, self.params
        return loss


def samples(counts, n_in, classes, device="cuda", seed=5):
    """Points around one centre a class; every worker sees the classes in a mix of its own."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    centres = torch.randn(classes, n_in, generator=g)
    xs, ys = [], []
    for n in counts:
        mix = torch.softmax(torch.randn(classes, generator=g) * 1.5, 0)
        y = torch.multinomial(mix, max(n, 1), replacement=True, generator=g)[:n]
        xs.append(centres[y] + torch.randn(n, n_in, generator=g) * 1.5)
        ys.append(y)
    return torch.cat(xs).to(device), torch.cat(ys).to(device)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--rounds", type=int, default=30)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--max-norm", type=float, default=1.0)
    ap.add_argument("--dropout", type=float, default=0.0)
    a = ap.parse_args(argv)
    counts = [100 + (37 * w) % 150 for w in range(a.workers)]
    dtype = torch.float32 if a.dtype == "f32" else torch.bfloat16
    x, y = samples(counts, 64, 10)
    w = Workers(counts, 64, 256, 10, 8, dtype, dropout=a.dropout)
    losses = []
    for r in range(a.rounds):
        loss = w.step(x.to(dtype), y, a.lr, a.max_norm, r, segments=4, replicas=min(2, a.workers - 1))
        losses.append(float(loss))
        if r % 5 == 0 or r + 1 == a.rounds:
            print("round %3d  loss %.4f  gradient norms %.3f to %.3f" % (r, losses[-1], float(w.norm.min()), float(w.norm.max())))
    combo.combo_device_status()
    return losses


if __name__ == "__main__":
    main()

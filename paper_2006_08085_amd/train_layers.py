"""A small network trained by the workers of a ring, each on its own unevenly drawn batches: the per-worker products, the
cross-entropy and AdamW together with a round of gossip.

    python -m paper_2006_08085_amd.train_layers [--workers 16] [--steps 200] [--bits 8]

Every worker keeps its own copy of a network with one hidden layer (64 -> 128 -> 10, relu) as a row of X (fp32), with a bfloat16
copy X16 that the products read.  A step, on n workers at once and without a word to the host:

    hidden = max(0, A W1^T)            linear            rows of all workers, one after the other; `rows` says whose are whose
    logits = hidden W2^T               linear
    dlogits, loss                      cross_entropy     mean over a worker's own rows
    G[W2], dhidden, G[W1]              linear_grad_weight, linear_grad_input
    X <- gossip(X)                     gossip_accel      K momentum rounds with the ring's neighbours
    X, X16 <- AdamW(X, G)              AdamW.step        moments in 32 bits or in 8

The data are points of ten overlapping classes; worker i draws half of its points from class i mod 10, and between 1 and 2 * --batch
points a step.  One JSON line per tenth of the run: mean loss, consensus distance, and the accuracy of the mean model on fresh
points of all classes.
"""
from __future__ import annotations

import argparse
import json

import torch

import paper_2006_08085_amd as D

INPUTS, HIDDEN, CLASSES = 64, 128, 10
W2 = HIDDEN * INPUTS                      # first column of the second layer
COLUMNS = W2 + CLASSES * HIDDEN


def train(workers: int = 16, steps: int = 200, bits: int = 8, batch: int = 32, lr: float = 2e-3, K: int = 2, seed: int = 1, records: int = 10):
    """Yields `records` dicts; the last holds the final state."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    ctx = D.detag_create(D.Topology.ring(), workers, COLUMNS, D.padded_ld(COLUMNS))
    one = D.detag_create(D.Topology.ring(), 1, COLUMNS, D.padded_ld(COLUMNS))        # the mean model
    opt = D.AdamW(ctx, [(0, W2), (W2, COLUMNS - W2)], weight_decay=[0.01, 0.01], bits=bits)
    most = 2 * batch * workers
    ctx.reserve_cross_entropy(most)
    centres = 0.45 * torch.randn(CLASSES, INPUTS, device=dev, generator=gen)

    def points(labels):
        return (centres[labels] + torch.randn(len(labels), INPUTS, device=dev, generator=gen)).bfloat16()

    X, G = D.new_matrix(workers, COLUMNS, device=dev), D.new_matrix(workers, COLUMNS, device=dev)
    X[:, :W2] = INPUTS ** -0.5 * torch.randn(W2, device=dev, generator=gen)        # all start from the same model
    X[:, W2:COLUMNS] = HIDDEN ** -0.5 * torch.randn(COLUMNS - W2, device=dev, generator=gen)
    X16 = X.bfloat16()
    M, V, S = opt.new_moments(dev)
    hidden, dhidden = (torch.empty(most, HIDDEN, dtype=torch.bfloat16, device=dev) for _ in range(2))
    logits, dlogits = (torch.empty(most, CLASSES, dtype=torch.bfloat16, device=dev) for _ in range(2))
    loss = torch.zeros(workers, device=dev)
    favourite = torch.arange(workers, device=dev) % CLASSES

    # all the batches' rows lie in matrices of `most` rows; those that no worker owns in a step are left alone
    rows = torch.zeros(workers + 1, dtype=torch.int32, device=dev)
    for t in range(1, steps + 1):
        rows[1:] = torch.randint(1, 2 * batch + 1, (workers,), device=dev, generator=gen).cumsum(0)
        owner = torch.searchsorted(rows[1:], torch.arange(most, dtype=torch.int32, device=dev), right=True).clamp_(max=workers - 1)
        any_class = torch.randint(CLASSES, (most,), device=dev, generator=gen)
        labels = torch.where(torch.rand(most, device=dev, generator=gen) < 0.5, favourite[owner], any_class)
        A, wanted = points(labels), labels.int()

        ctx.linear(X16, 0, A, rows, hidden, relu=True)
        ctx.linear(X16, W2, hidden, rows, logits)
        ctx.cross_entropy(logits, wanted, rows, dlogits, loss)
        ctx.linear_grad_weight(dlogits, hidden, rows, G, W2)
        ctx.linear_grad_input(X16, W2, dlogits, rows, dhidden, relu_of=hidden)
        ctx.linear_grad_weight(dhidden, A, rows, G, 0)
        ctx.gossip_accel(X, K)
        # with 8 bits a second moment may be kept as zero: the limit holds such a step back
        opt.step(X, G, M, V, S, lr=lr, t=t, seed=seed, limit=4.0 if bits == 8 else 0.0, X16=X16)

        if t % max(1, steps // records) == 0 or t == steps:
            fresh = torch.arange(2000, device=dev) % CLASSES
            mean = torch.zeros(1, one.ld, device=dev)
            mean[0, :COLUMNS] = ctx.mean(X)[:COLUMNS]
            all_rows = torch.tensor([0, len(fresh)], dtype=torch.int32, device=dev)
            h, z = (torch.empty(len(fresh), c, dtype=torch.bfloat16, device=dev) for c in (HIDDEN, CLASSES))
            one.linear(mean.bfloat16(), 0, points(fresh), all_rows, h, relu=True)
            one.linear(mean.bfloat16(), W2, h, all_rows, z)
            yield {"step": t, "workers": workers, "bits": bits, "loss": float(loss.mean()), "consensus_distance": float(ctx.consensus_error(X)),
                   "accuracy_of_mean_model": float((z.argmax(1) == fresh).float().mean())}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workers", type=int, default=16)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    args = ap.parse_args()
    for row in train(args.workers, args.steps, args.bits):
        print(json.dumps(row))


if __name__ == "__main__":
    main()

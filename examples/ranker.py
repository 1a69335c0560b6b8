"""A small ranker on one GPU: the embedding lookup, then the dense layers that turn its pooled rows into a score.

    pooled = lookup(indices, offsets)                 [B, T * E], fp32
    x = relu(pooled W0^T + b0) + relu(dense Wd^T + bd)
    x = x + (silu(x Wg^T) * (x Wu^T)) Wo^T + bo       a gated feed-forward block with a skip connection
    score = sigmoid(x Ws^T + bs)

``Ranker.scores`` serves; ``Ranker.train_step`` takes one step of gradient descent on the logistic loss (the tables stay
as they are).  Run as a script it does both on seeded synthetic queries:

    python examples/ranker.py [--dtype f32|f16|bf16] [--batch 4096] [--steps 50]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_01676_amd as embx  # noqa: E402
import workloads as W  # noqa: E402

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Ranker:
    """``rows``: rows of each table.  Weights are held in ``dtype``, the type of the dense layers."""

    def __init__(self, rows, E, stats, max_batch, *, dense=13, width=256, inner=704, dtype="bf16", seed=0):
        self.dtype = DTYPES[dtype]
        self.plan = embx.Plan(rows, E, "f32", stats, max_batch)
        tables = []
        for t, m in enumerate(rows):
            tables.append(torch.empty((m, E), dtype=torch.float32, device="cuda"))
            embx.fill_table(tables[-1], t, seed + t)
        self.plan.bind(tables)
        gen = torch.Generator().manual_seed(seed)
        k = len(rows) * E

        def weight(n, k_):
            return (torch.randn(n, k_, generator=gen) * k_ ** -0.5).to(self.dtype).cuda()

        def bias(n):
            return torch.zeros(n, dtype=self.dtype, device="cuda")

        self.p = {"w0": weight(width, k), "b0": bias(width), "wd": weight(width, dense), "bd": bias(width),
                  "wg": weight(inner, width), "wu": weight(inner, width), "wo": weight(width, inner), "bo": bias(width),
                  "ws": weight(1, width), "bs": bias(1)}

    def pooled(self, indices, offsets, batch):
        # the lookup's fp32 sums, scaled to order one, in the type of the layers
        out = self.plan.lookup(indices, offsets, batch)
        return (out.view(batch, -1) * 10.0).to(self.dtype)

    def scores(self, indices, offsets, dense):
        """[B] probabilities, in the type of the layers."""
        p, batch = self.p, dense.shape[0]
        side = embx.linear(dense, p["wd"], p["bd"], activation="relu")
        x = embx.linear(self.pooled(indices, offsets, batch), p["w0"], p["b0"], side, activation="relu")
        h = embx.gated_ffn(x, p["wg"], p["wu"])
        x = embx.linear(h, p["wo"], p["bo"], x)
        return embx.linear(x, p["ws"], p["bs"], activation="sigmoid").view(-1)

    def gradients(self, indices, offsets, dense, labels):
        """(loss, gradients by name): the mean logistic loss over the batch."""
        p, batch = self.p, dense.shape[0]
        pooled = self.pooled(indices, offsets, batch)
        side, z_side = embx.linear(dense, p["wd"], p["bd"], activation="relu", save=True)
        x0, z0 = embx.linear(pooled, p["w0"], p["b0"], side, activation="relu", save=True)
        h, g, u = embx.gated_ffn(x0, p["wg"], p["wu"], save=True)
        x1 = embx.linear(h, p["wo"], p["bo"], x0)
        score, z = embx.linear(x1, p["ws"], p["bs"], activation="sigmoid", save=True)
        loss = torch.nn.functional.binary_cross_entropy_with_logits(z.float().view(-1), labels)
        # of the loss by z: score - label; summed here over the batch, divided by it in the step
        dz = (score.float().view(-1) - labels).to(self.dtype).view(-1, 1)
        d = {}
        dx1, d["ws"], d["bs"] = embx.linear_backward(dz, x1, p["ws"])
        dh, d["wo"], d["bo"] = embx.linear_backward(dx1, h, p["wo"])
        dx0, d["wg"], d["wu"], _, _ = embx.gated_ffn_backward(dh, x0, p["wg"], p["wu"], g, u)
        dx0 += dx1   # the skip connection
        _, d["w0"], d["b0"] = embx.linear_backward(dx0, pooled, p["w0"], z0, activation="relu", need_dx=False)
        _, d["wd"], d["bd"] = embx.linear_backward(dx0, dense, p["wd"], z_side, activation="relu", need_dx=False)
        return loss, d

    def train_step(self, indices, offsets, dense, labels, rate=0.1):
        """One step; returns the loss before it (a device scalar)."""
        loss, d = self.gradients(indices, offsets, dense, labels)
        for name, grad in d.items():
            self.p[name].add_(grad, alpha=-rate / dense.shape[0])
        return loss


def queries(rows, batch, seed, dtype, dense=13, pooling=8):
    """Seeded synthetic queries: (indices, offsets, dense features, labels that depend on the features)."""
    gen = torch.Generator().manual_seed(seed)
    indices = torch.cat([torch.randint(0, m, (batch * pooling,), generator=gen) for m in rows])
    offsets = torch.arange(len(rows) * batch + 1, dtype=torch.int64) * pooling
    features = torch.randn(batch, dense, generator=gen)
    labels = (features[:, 0] + 0.5 * features[:, 1] > 0).float()
    return indices.cuda(), offsets.cuda(), features.to(DTYPES[dtype]).cuda(), labels.cuda()


def make(rows, E, batch, dtype, **kw):
    stats = [W.TableStats(mean_pooling=8.0, max_pooling=8, hot_rows=[], hot_freq=[], unique_frac=1.0) for _ in rows]
    return Ranker(rows, E, stats, batch, dtype=dtype, **kw)


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--dtype", choices=DTYPES, default="bf16")
    a.add_argument("--batch", type=int, default=4096)
    a.add_argument("--steps", type=int, default=50)
    a = a.parse_args()
    rows, E = [100000] * 26, 64
    r = make(rows, E, a.batch, a.dtype)
    q = queries(rows, a.batch, 1, a.dtype)
    for step in range(a.steps):
        loss = r.train_step(*q)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {loss.item():.4f}", flush=True)
    scores = r.scores(*q[:3])
    right = ((scores.float() > 0.5).float() == q[3]).float().mean().item()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(100):
        r.scores(*q[:3])
    torch.cuda.synchronize()
    print(f"{right:.1%} of {a.batch} labels right; {(time.perf_counter() - start) * 1e4:.0f} us a batch of scores")


if __name__ == "__main__":
    main()

"""One training step of a graph model on the library's own operators.

A learned table E (one row per node) is aggregated over the graph, normalised
and scored against classes:

    Z = A E,  Y = layer norm(Z),  loss = cross entropy(Y W^T, labels)

and backwards: dY, dW from the loss, dZ, dgamma, dbeta from the norm, dE = A dZ
(A is symmetric), then AdamW over all four tensors, the table's moments held in
8 bits.  Every step of the arithmetic is one of the library's calls; torch
holds the memory.  Labels follow the graph: a node has the class of the
community that it belongs to, and a tenth of the nodes have none.

    python examples/node_classification.py [--nodes 20000] [--steps 60]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_02006_amd as aires  # noqa: E402


def communities(n, classes, degree, seed):
    """A symmetric graph with self-loops whose edges stay within a node's class
    four times in five, its values 1/sqrt(d_i d_j), and the classes."""
    rng = np.random.default_rng(seed)
    of = rng.integers(0, classes, n)
    members = [np.flatnonzero(of == c) for c in range(classes)]
    src = np.repeat(np.arange(n), degree // 2)
    inside = rng.random(src.size) < 0.8
    dst = rng.integers(0, n, src.size)
    for c in range(classes):
        pick = inside & (of[src] == c)
        dst[pick] = rng.choice(members[c], pick.sum())
    keys = np.unique(np.concatenate([src * n + dst, dst * n + src, np.arange(n) * (n + 1)]))
    row, col = keys // n, keys % n
    d = np.bincount(row, minlength=n)
    rp = np.concatenate([[0], np.cumsum(d)]).astype(np.int64)
    val = (1 / np.sqrt(d[row] * d[col])).astype(np.float32)
    return (n, n, rp, col.astype(np.int32), val), of


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--nodes", type=int, default=20000)
    ap.add_argument("--features", type=int, default=64)
    ap.add_argument("--classes", type=int, default=12)
    ap.add_argument("--degree", type=int, default=16)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=0.02)
    a = ap.parse_args(argv)
    graph, of = communities(a.nodes, a.classes, a.degree, 1)
    A = aires.to_device(graph)
    labels = torch.from_numpy(of).cuda()
    held = torch.from_numpy(np.random.default_rng(2).random(a.nodes) < 0.1).cuda()
    train = torch.where(held, torch.full_like(labels, -1), labels)

    g = torch.Generator(device="cuda").manual_seed(3)
    E = 0.1 * torch.randn((a.nodes, a.features), generator=g, device="cuda")
    gamma, beta = torch.ones(a.features, device="cuda"), torch.zeros(a.features, device="cuda")
    W = 0.1 * torch.randn((a.classes, a.features), generator=g, device="cuda")
    params = [E, gamma, beta, W]
    m8, v8 = aires.adamw_state([E], bits=8)        # the table: 2 bytes a value, not 8
    m32, v32 = aires.adamw_state(params[1:])
    m, v = m8 + m32, v8 + v32

    losses = []
    for step in range(1, a.steps + 1):
        Z = aires.spmm(A, E)
        Y, mean, rstd = aires.layer_norm(Z, gamma, beta)
        x = aires.linear_xent(Y, W, train)
        dZ, dgamma, dbeta = aires.layer_norm_backward(x.dH, Z, mean, rstd, gamma)
        dE = aires.spmm(A, dZ)
        aires.adamw(params, [dE, dgamma, dbeta, x.dW], m, v, step=step, lr=a.lr, weight_decay=0.0, seed=step)
        losses.append(x.loss)
    losses = torch.stack(losses).tolist()          # the only copies to the host

    Y, _, _ = aires.layer_norm(aires.spmm(A, E), gamma, beta, stats=False)
    test = aires.linear_xent(Y, W, torch.where(held, labels, torch.full_like(labels, -1)), grads=False)
    right = ((Y @ W.t()).argmax(1) == labels)[held].float().mean()
    print("loss %.4f -> %.4f; held-out nodes: loss %.4f, %.1f %% right" %
          (losses[0], losses[-1], float(test.loss), 100 * float(right)))
    return losses, float(test.loss), float(right)


if __name__ == "__main__":
    main()

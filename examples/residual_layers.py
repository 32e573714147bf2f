"""Residual layers on aggregated node features, with products in 8 bits.

The features of a graph's nodes are aggregated once and go through layers that each
add to a residual stream,

    s = x + r,  y = rms norm(s),  x' = y W^T,

and the last norm's output is scored against classes.  y and W are held in 8 bits
for the products: y with a scale for each 128 values of a row, W for each 128 x
128 values, dy likewise on the way back; a weight's gradient sums over the nodes
and takes both operands with scales along them.  The loss is the mean negative log
probability of the labels, less a little of the entropy (which keeps the answers
from becoming certain too early).  All gradients together are clipped to a norm,
whose factor the update reads on the device.  Every step of the arithmetic is one
of the library's calls; torch holds the memory.

    python examples/residual_layers.py [--nodes 20000] [--steps 60]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_02006_amd as aires  # noqa: E402
from examples.node_classification import communities  # noqa: E402

BF16 = torch.bfloat16


def model(features, classes, layers, seed=3):
    """Weights in fp32: for each layer and for the scores gamma and W."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    shapes = [(features, features)] * layers + [(classes, features)]
    return [p for out, d in shapes for p in
            (torch.ones(d, device="cuda"), torch.randn((out, d), generator=g, device="cuda") * d ** -0.5)]


def forward(params, x):
    """Scores (fp32) of the rows of x (bf16), and what the way back needs."""
    kept, r = [], None
    for k in range(0, len(params), 2):
        gamma, W = params[k:k + 2]
        y, s, rstd = aires.rms_norm(x, gamma, residual=r)
        s = x if s is None else s
        y8, y8t = aires.quantize_8bit(y, order="both")
        W8, W8t = aires.quantize_8bit(W, tiles=True, order="both")
        last = k == len(params) - 2
        x = aires.matmul_8bit(y8, W8, out_dtype=torch.float32 if last else BF16)
        kept.append(dict(s=s, rstd=rstd, y8=y8, y8t=y8t, W8=W8, W8t=W8t, out=x))
        r = s
    return x, kept


def backward(params, kept, dz):
    """Gradients of all weights and of the rows, from those of the scores."""
    grads, dx, ds = [None] * len(params), dz, None
    for k in reversed(range(0, len(params), 2)):
        c = kept[k // 2]
        c["dx8"], c["dx8t"] = aires.quantize_8bit(dx, order="both")
        grads[k + 1] = aires.matmul_8bit(c["dx8t"], c["y8t"], out_dtype=torch.float32)
        c["dy"] = aires.matmul_8bit(c["dx8"], c["W8t"])
        # what reaches the stream past this layer's norm comes from the next layer's
        c["ds"] = ds
        ds, grads[k] = aires.rms_norm_backward(c["dy"], c["s"], c["rstd"], params[k], dS=ds)
        dx = ds
    return grads, ds


def loss_and_gradient(z, labels, entropy_weight):
    """-(sum of log probabilities + w entropy) / number of labels, and dz."""
    r = aires.log_probs(z, labels, rest=True)
    there = labels >= 0
    count = there.sum().clamp(min=1)
    loss = -(r.logp.sum() + entropy_weight * (r.entropy * there).sum()) / count
    dlogp = -(there / count).float()
    dz = aires.log_probs_backward(z, labels, r.lse, r.entropy, lse_rest=r.lse_rest, dlogp=dlogp,
                                  dentropy=entropy_weight * dlogp)
    return loss, dz


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--nodes", type=int, default=20000)
    ap.add_argument("--features", type=int, default=256)
    ap.add_argument("--classes", type=int, default=12)
    ap.add_argument("--degree", type=int, default=16)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--lr", type=float, default=3e-3)
    a = ap.parse_args(argv)
    graph, of = communities(a.nodes, a.classes, a.degree, 1)
    rng = np.random.default_rng(2)
    X = rng.standard_normal((a.nodes, a.features)) + 0.5 * rng.standard_normal((a.classes, a.features))[of]
    x = aires.spmm(aires.to_device(graph), torch.from_numpy(X.astype(np.float32)).cuda()).to(BF16)
    labels = torch.from_numpy(of).cuda()
    held = torch.from_numpy(rng.random(a.nodes) < 0.1).cuda()
    train = torch.where(held, torch.full_like(labels, -1), labels)

    params = model(a.features, a.classes, a.layers)
    m, v = aires.adamw_state(params)
    losses, norms = [], []
    for step in range(1, a.steps + 1):
        z, kept = forward(params, x)
        loss, dz = loss_and_gradient(z, train, 0.01)
        grads, _ = backward(params, kept, dz)
        norm, scale = aires.grad_norm(grads, max_norm=1.0)
        aires.adamw(params, grads, m, v, step=step, lr=a.lr, weight_decay=0.0, grad_scale=scale)
        losses.append(loss)
        norms.append(norm)
    losses = torch.stack(losses).tolist()          # the only copies to the host
    z, _ = forward(params, x)
    r = aires.log_probs(z, labels, top=min(3, a.classes))
    first = (r.top_index[:, 0] == labels)[held].float().mean()
    some = (r.top_index == labels[:, None]).any(1)[held].float().mean()
    print("loss %.4f -> %.4f (gradient norm %.3f -> %.3f); held-out nodes: %.1f %% right, %.1f %% among three, entropy %.3f" %
          (losses[0], losses[-1], float(norms[0]), float(norms[-1]), 100 * float(first), 100 * float(some),
           float(r.entropy[held].mean())))
    return losses, float(first)


if __name__ == "__main__":
    main()

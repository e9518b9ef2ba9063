"""Trains a small encoder of graph nodes with this library's operators and compares graphs by transport.

Nodes of ragged graphs go through a tanh layer, attention inside their own graph (near nodes of the order count more)
and a linear layer with the residual, and with --hidden through a gated feed-forward block behind a layer norm; the loss
is the cross entropy of every node against a vocabulary of prototypes at scale 1 / lambda.  The gradients are formed by the
operators' backward calls, layer by layer, and applied by plain gradient descent, with --orthogonal those of matrices with
their singular values brought to 0.7 .. 1.2.  At the end the encoded graphs of every pair are compared by a batch of
transport problems.

    python examples/train_encoder.py [--graphs 64] [--steps 60] [--bf16] [--hidden 64] [--orthogonal]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2107_06876_amd as lcn  # noqa: E402


class Encoder:
    """tanh layer, attention inside the sets, linear layer with residual; with `hidden` also a layer norm, a gated layer that
    wide, and the linear layer back with its residual.  Keeps what its backward pass needs."""

    def __init__(self, d_in, d, heads, dtype, device, seed=1, hidden=0):
        g = torch.Generator(device="cpu")
        g.manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=g) * cols ** -0.5).to(dtype).to(device)

        self.heads, self.dim = heads, d // heads
        self.weights = dict(w1=matrix(d, d_in), b1=torch.zeros(d, dtype=dtype, device=device), wqkv=matrix(3 * d, d),
                            wo=matrix(d, d), bo=torch.zeros(d, dtype=dtype, device=device))
        self.hidden = hidden
        if hidden:
            self.weights.update(norm=torch.ones(d, dtype=dtype, device=device), shift=torch.zeros(d, dtype=dtype, device=device),
                                wg=matrix(2 * hidden, d), bg=torch.zeros(2 * hidden, dtype=dtype, device=device), wd=matrix(d, hidden))
        self.slopes = (2.0 ** -torch.arange(1, heads + 1).float()).to(device)

    def forward(self, x, offsets):
        p, n = self.weights, x.shape[0]
        h, pre = lcn.lcn_linear(x, p["w1"], bias=p["b1"], activation=lcn.ACT_TANH, keep_pre=True)
        qkv = lcn.lcn_linear(h, p["wqkv"]).view(n, 3, self.heads, self.dim)
        o, lse = lcn.lcn_attention(qkv[:, 0], qkv[:, 1], qkv[:, 2], offsets, offsets, slopes=self.slopes)
        y = lcn.lcn_linear(o.view(n, -1), p["wo"], bias=p["bo"], residual=h)
        self.kept = (x, offsets, h, pre, qkv, o, lse)
        if not self.hidden:
            return y
        m, mean, rstd = lcn.lcn_layer_norm(y, p["norm"], p["shift"], keep_stats=True)
        f, gates = lcn.lcn_gated_linear(m, p["wg"], bias=p["bg"], activation=lcn.ACT_SILU, keep_pre=True)
        self.kept_block = (y, m, mean, rstd, f, gates)
        return lcn.lcn_linear(f, p["wd"], residual=y)

    def backward(self, dy):
        """The gradients of the weights for a given dy, and that of x."""
        p = self.weights
        x, offsets, h, pre, qkv, o, lse = self.kept
        n, block = x.shape[0], {}
        if self.hidden:
            y, m, mean, rstd, f, gates = self.kept_block
            df, dwd, _ = lcn.lcn_linear_backward(f, p["wd"], None, dy, with_bias=False)
            dm, dwg, dbg = lcn.lcn_gated_linear_backward(m, p["wg"], gates, df, activation=lcn.ACT_SILU)
            dy, dnorm, dshift = lcn.lcn_layer_norm_backward(y, p["norm"], mean, rstd, dm, around=dy)
            block = dict(norm=dnorm, shift=dshift, wg=dwg, bg=dbg, wd=dwd)
        do, dwo, dbo = lcn.lcn_linear_backward(o.view(n, -1), p["wo"], None, dy)
        dq, dk, dv = lcn.lcn_attention_backward(qkv[:, 0], qkv[:, 1], qkv[:, 2], o, lse, do.view_as(o), offsets, offsets,
                                                slopes=self.slopes)
        dh, dwqkv, _ = lcn.lcn_linear_backward(h, p["wqkv"], None, torch.stack((dq, dk, dv), dim=1).view(n, -1),
                                               with_bias=False)
        dh += dy   # the residual
        dx, dw1, db1 = lcn.lcn_linear_backward(x, p["w1"], pre, dh, activation=lcn.ACT_TANH)
        return dict(w1=dw1, b1=db1, wqkv=dwqkv, wo=dwo, bo=dbo, **block), dx


def graphs(count, d_in, classes, device, dtype, seed=2):
    """Ragged graphs of 16 to 64 nodes: noisy copies of class prototypes, and every node's class."""
    rng = np.random.default_rng(seed)
    sizes = rng.integers(16, 65, size=count)
    target = rng.integers(0, classes, size=int(sizes.sum()))
    centres = rng.standard_normal((classes, d_in))
    x = centres[target] + 0.5 * rng.standard_normal((len(target), d_in))
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    return (torch.from_numpy(x).to(dtype).to(device), torch.from_numpy(offsets).to(device), offsets,
            torch.from_numpy(target).to(device))


def train(count=64, steps=30, d_in=32, d=32, heads=4, classes=1000, lam=0.5, rate=0.05, dtype=torch.float32,
          device="cuda:0", say=print, hidden=0, orthogonal=False):
    """Returns (losses of all steps, transport distances of the pairs (2 p, 2 p + 1))."""
    x, off, host_off, target = graphs(count, d_in, classes, device, dtype)
    model = Encoder(d_in, d, heads, dtype, device, hidden=hidden)
    g = torch.Generator(device="cpu")
    g.manual_seed(3)
    vocabulary = (torch.randn(classes, d, generator=g) * d ** -0.5).to(dtype).to(device)
    weight = torch.full((x.shape[0],), 1.0 / x.shape[0], device=device)
    losses = []
    for step in range(steps):
        y = model.forward(x, off)
        loss, lse = lcn.lcn_cross_entropy(y, vocabulary, target, scale=1.0 / lam)
        dy, dvoc, _ = lcn.lcn_cross_entropy_backward(y, vocabulary, target, lse, weight, scale=1.0 / lam)
        grads, _ = model.backward(dy)
        for name, w in model.weights.items():
            step_of = grads[name]
            if orthogonal and w.dim() == 2:   # of the size of the weights' own rows
                step_of = lcn.lcn_orthogonalise(step_of, scale=0.2 * max(w.shape) ** 0.5)
            w -= (rate * step_of.float()).to(w.dtype)
        # a word is the target of one row in `classes`: its gradient is so much smaller
        vocabulary -= (0.1 * rate * classes * dvoc.float()).to(vocabulary.dtype)
        losses.append(float((loss * weight).sum()))
        if step % 10 == 0 or step == steps - 1:
            say("step %d: loss %.4f" % (step, losses[-1]), flush=True)
    # encoded graphs 2 p and 2 p + 1 are compared by transport with deletion rows and columns
    y = model.forward(x, off).float()
    pairs = count // 2
    left = [torch.arange(host_off[2 * p], host_off[2 * p + 1]) for p in range(pairs)]
    right = [torch.arange(host_off[2 * p + 1], host_off[2 * p + 2]) for p in range(pairs)]
    X, Y = y[torch.cat(left).to(device)].contiguous(), y[torch.cat(right).to(device)].contiguous()
    ends = [np.concatenate([[0], np.cumsum([len(t) for t in side])]).astype(np.int64) for side in (left, right)]
    ones = [torch.ones(t.shape[0], device=device) for t in (X, Y)]
    h = lcn.lcn_build_batched(X, Y, ends[0], ends[1], np.full(pairs, lam, dtype=np.float32), lcn.COST_EUCLID, lcn.MODE_DENSE,
                              del_cost_x=ones[0], del_cost_y=ones[1])
    lcn.sinkhorn_run(h, 50)
    distances, _ = lcn.lcn_batched_results(h)
    say("transport distances of %d pairs: %.4f .. %.4f" % (pairs, distances.min(), distances.max()), flush=True)
    return losses, distances


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--graphs", type=int, default=64)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--bf16", action="store_true")
    ap.add_argument("--hidden", type=int, default=0)
    ap.add_argument("--orthogonal", action="store_true")
    a = ap.parse_args()
    train(a.graphs, a.steps, dtype=torch.bfloat16 if a.bf16 else torch.float32, hidden=a.hidden, orthogonal=a.orthogonal)

"""The operators together: examples/train_encoder.py learns, and its hand-written backward pass is the gradient of its
forward pass (against automatic differentiation of the same formulas in 64 bits)."""
import os
import sys

import numpy as np
import pytest
import torch

from operator_checks import BF16, DEV, F32, bound, off

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_gradients_of_the_whole_encoder():
    import train_encoder as ex
    x, offsets, host, _ = ex.graphs(6, 32, 50, DEV, F32)
    model = ex.Encoder(32, 32, 4, F32, DEV)
    y = model.forward(x, offsets)
    dy = torch.randn(y.shape, generator=torch.Generator().manual_seed(4)).to(DEV)
    grads, dx = model.backward(dy)
    p = {k: w.double().cpu().requires_grad_(True) for k, w in model.weights.items()}
    X = x.double().cpu().requires_grad_(True)
    h = torch.tanh(X @ p["w1"].t() + p["b1"])
    qkv = (h @ p["wqkv"].t()).view(len(X), 3, 4, 8)
    rows = []
    for a, b in zip(host[:-1], host[1:]):
        q, k, v = (qkv[a:b, i].permute(1, 0, 2) for i in range(3))
        far = (torch.arange(b - a)[:, None] - torch.arange(b - a)[None, :]).abs()
        z = q @ k.transpose(1, 2) / 8 ** 0.5 - model.slopes.double().cpu()[:, None, None] * far
        rows.append((torch.softmax(z, 2) @ v).permute(1, 0, 2).reshape(b - a, 32))
    out = torch.cat(rows) @ p["wo"].t() + p["bo"] + h
    out.backward(dy.double().cpu())
    # three products deep, each with the error of its own sums
    assert off(y.cpu(), out.detach()) <= 4 * bound(F32, 64)
    for name, w in p.items():
        assert off(grads[name].cpu(), w.grad) <= 16 * bound(F32, len(X))
    assert off(dx.cpu(), X.grad) <= 16 * bound(F32, 64)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_example_learns(dtype):
    import train_encoder as ex
    losses, distances = ex.train(count=32, steps=20, dtype=dtype)
    assert np.isfinite(losses).all() and np.isfinite(distances).all()
    assert losses[-1] < 0.9 * losses[0]

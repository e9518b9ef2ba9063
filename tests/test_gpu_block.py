"""The operators of a layer together: layer norm, gated layer and linear layer with its residual behind the attention of
examples/train_encoder.py, their gradients against automatic differentiation of the same formulas in 64 bits, and a training step
with orthogonalised updates, eager, captured, and two at once."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, generator, normal, off

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden", [48, 96, 37])
def test_gradients_of_the_whole_encoder(hidden):
    import train_encoder as ex
    x, offsets, host, _ = ex.graphs(6, 32, 50, DEV, F32)
    model = ex.Encoder(32, 32, 4, F32, DEV, hidden=hidden)
    g = generator(hidden)
    for name in ("norm", "shift", "bg"):
        model.weights[name] += 0.3 * torch.randn(model.weights[name].shape, generator=g).to(DEV)
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
    s = torch.cat(rows) @ p["wo"].t() + p["bo"] + h
    c = s - s.mean(1, keepdim=True)
    m = c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * p["norm"] + p["shift"]
    z = m @ p["wg"].t() + p["bg"]
    gate = z[:, :hidden]
    out = gate / (1.0 + torch.exp(-gate)) * z[:, hidden:] @ p["wd"].t() + s
    out.backward(dy.double().cpu())
    # six products deep, each with the error of its own sums
    assert off(y.cpu(), out.detach()) <= 8 * bound(F32, 64)
    assert set(grads) == set(p)
    for name, w in p.items():
        assert off(grads[name].cpu(), w.grad) <= 32 * bound(F32, len(X))
    assert off(dx.cpu(), X.grad) <= 32 * bound(F32, 64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("orthogonal", [False, True])
def test_the_example_runs(orthogonal, dtype):
    import train_encoder as ex
    losses, distances = ex.train(count=16, steps=4, dtype=dtype, hidden=64, orthogonal=orthogonal)
    assert np.isfinite(losses).all() and np.isfinite(distances).all()


class Block:
    """x + Wd (act(m Wg^T) (m Wu^T)), m the norm of x, and one update of its weights from a given gradient."""

    def __init__(self, rows, d, hidden, dtype, key):
        g = generator(rows, d, hidden, key)
        self.x, self.dy = normal(g, rows, d, dtype=dtype), normal(g, rows, d, dtype=dtype)
        self.norm, self.shift = 1.0 + normal(g, d, dtype=dtype, scale=0.1), normal(g, d, dtype=dtype, scale=0.1)
        self.w, self.wd = normal(g, 2 * hidden, d, dtype=dtype, scale=d ** -0.5), normal(g, d, hidden, dtype=dtype, scale=hidden ** -0.5)

    def step(self):
        m, mean, rstd = lcn.lcn_layer_norm(self.x, self.norm, self.shift, keep_stats=True)
        f, kept = lcn.lcn_gated_linear(m, self.w, keep_pre=True)
        y = lcn.lcn_linear(f, self.wd, residual=self.x)
        df, dwd, _ = lcn.lcn_linear_backward(f, self.wd, None, self.dy, with_bias=False)
        dm, dw, _ = lcn.lcn_gated_linear_backward(m, self.w, kept, df, with_bias=False)
        dx, dnorm, dshift = lcn.lcn_layer_norm_backward(self.x, self.norm, mean, rstd, dm, around=self.dy)
        new_w = self.w + lcn.lcn_orthogonalise(dw, scale=-0.02)
        new_wd = self.wd + lcn.lcn_orthogonalise(dwd, scale=-0.02)
        return y, dx, dnorm, dshift, new_w, new_wd


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d,hidden", [(1, 64, 96), (700, 32, 64), (900, 300, 128), (515, 128, 600)])
def test_a_step_captured(rows, d, hidden, dtype):
    block = Block(rows, d, hidden, dtype, 1)
    want = block.step()
    assert all(torch.isfinite(t).all() for t in want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        block.step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block.step()
    keep = block.x.clone()
    for scale in (1.0, 0.5, 1.0):   # other inputs between replays, and eager work of the same kind
        block.x.copy_(keep * scale)
        want = block.step()
        for t in got:
            t.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, want):
            assert torch.equal(u, v)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_two_steps_at_once(dtype):
    """Calls on two streams, each with workspaces of its own, give the bits that they give alone."""
    blocks = [Block(900, 300, 128, dtype, 1), Block(700, 256, 260, dtype, 2)]
    want = [b.step() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = [None, None]
    for _ in range(5):
        for i, (b, s) in enumerate(zip(blocks, streams)):
            with torch.cuda.stream(s):
                got[i] = b.step()
    torch.cuda.synchronize()
    for u, v in zip(got, want):
        for a, b in zip(u, v):
            assert torch.equal(a, b)


def test_a_workspace_of_the_callers():
    """A workspace with anything in it, as large as the call says, and nothing behind it is touched."""
    x, w = torch.randn(300, 72, device=DEV).bfloat16(), torch.randn(400, 72, device=DEV).bfloat16()
    dy, g = torch.randn(300, 200, device=DEV).bfloat16(), torch.randn(2, 300, 200, device=DEV)
    y, kept = lcn.lcn_gated_linear(x, w, keep_pre=True)
    n, mean, rstd = lcn.lcn_layer_norm(x, keep_stats=True)
    from paper_2107_06876_amd import encoder
    calls = (("lcn_gated_linear_workspace_bytes", (300, 72, 200, 1, 0), lambda s: (lcn.lcn_gated_linear(x, w, workspace=s),)),
             ("lcn_gated_linear_workspace_bytes", (300, 72, 200, 1, 1), lambda s: lcn.lcn_gated_linear_backward(x, w, kept, dy, workspace=s)),
             ("lcn_layer_norm_workspace_bytes", (300, 72, 1), lambda s: lcn.lcn_layer_norm_backward(x, None, mean, rstd, n, workspace=s)),
             ("lcn_orthogonalise_workspace_bytes", (2, 300, 200, 0), lambda s: (lcn.lcn_orthogonalise(g, workspace=s),)))
    for name, sizes, f in calls:
        need = encoder._bytes(name, sizes)
        assert need > 0
        want = f(None)
        for fill in (0, 255, 127):
            space = torch.full((need + 4096,), fill, dtype=torch.uint8, device=DEV)
            for a, b in zip(f(space[:need]), want):
                assert torch.equal(a, b)
            assert (space[need:] == fill).all()


# ---- offsets beyond 32 bits -------------------------------------------------------


def test_norm_of_more_than_2_to_31_values():
    rows, dim = (1 << 21) + 5, 1024
    x = torch.empty(rows, dim, dtype=BF16, device=DEV)
    x[-3000:] = torch.randn(3000, dim, device=DEV).bfloat16()
    x[:-3000] = x[-3000:].repeat(rows // 3000 + 1, 1)[:rows - 3000]
    y, mean, rstd = lcn.lcn_layer_norm(x, keep_stats=True)
    assert torch.equal(y[-3000:], lcn.lcn_layer_norm(x[-3000:].contiguous()))
    dx, dw, db = lcn.lcn_layer_norm_backward(x, None, mean, rstd, y)
    few = lcn.lcn_layer_norm_backward(x[-3000:].contiguous(), None, mean[-3000:].contiguous(), rstd[-3000:].contiguous(),
                                      y[-3000:].contiguous())
    assert torch.equal(dx[-3000:], few[0])
    assert torch.isfinite(dw).all()


def test_gated_layer_of_more_than_2_to_31_values():
    rows, d_in, d_out = 600011, 64, 2048
    x = torch.randn(rows, d_in, device=DEV).bfloat16()
    w = (torch.randn(2 * d_out, d_in, device=DEV) / 8).bfloat16()
    y, kept = lcn.lcn_gated_linear(x, w, keep_pre=True)
    last = x[-4000:].contiguous()
    few, few_kept = lcn.lcn_gated_linear(last, w, keep_pre=True)
    assert off(y[-4000:], few.double()) <= 2.0 ** -8
    dy = torch.randn(rows, d_out, device=DEV).bfloat16()
    dx, _, _ = lcn.lcn_gated_linear_backward(x, w, kept, dy, with_bias=False, with_w=False)
    few_dx, _, _ = lcn.lcn_gated_linear_backward(last, w, few_kept, dy[-4000:].contiguous(), with_bias=False, with_w=False)
    # the same product rounded twice, of dz rounded twice
    assert off(dx[-4000:], few_dx.double()) <= 2 * 2.0 ** -8


@pytest.mark.parametrize("count,rows,cols", [(2050, 1024, 1024), (140000, 128, 124)])
def test_more_than_2_to_31_values_of_matrices(count, rows, cols):
    one = torch.randn(16, rows, cols, device=DEV).bfloat16()
    g = one.repeat((count + 15) // 16, 1, 1)[:count]
    want = lcn.lcn_orthogonalise(one, steps=2)
    x = lcn.lcn_orthogonalise(g, steps=2, out=g)
    for i in (0, 1, count // 2, count - 1):
        assert off(x[i], want[i % 16].double()) <= 2.0 ** -8

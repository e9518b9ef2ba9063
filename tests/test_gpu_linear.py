"""lcn_linear and lcn_linear_backward against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, generator, normal, off

pytestmark = pytest.mark.gpu

ACTS = {"none": lcn.ACT_NONE, "tanh": lcn.ACT_TANH, "relu": lcn.ACT_RELU, "gelu": lcn.ACT_GELU, "silu": lcn.ACT_SILU}
FUNCTIONS = dict(none=lambda z: z * 1.0, tanh=torch.tanh, relu=torch.relu, gelu=torch.nn.functional.gelu,
                 silu=torch.nn.functional.silu)


def oracle(x, w, b, r, dy, act):
    """y, z, dx, dw, db in 64 bits."""
    x, w, dy = x.double(), w.double(), dy.double()
    z = x @ w.t().contiguous()
    if b is not None:
        z = z + b.double()
    z = z.detach().requires_grad_(True)
    y = FUNCTIONS[act](z)
    (dz,) = torch.autograd.grad(y, z, dy)
    y = y.detach() + (r.double() if r is not None else 0.0)
    return y, z.detach(), dz @ w, dz.t().contiguous() @ x, dz.sum(0)


def check(rows, d_in, d_out, act, dtype, bias=True, residual=True, shift=0):
    print("linear", rows, d_in, d_out, act, dtype, bias, residual, shift, flush=True)
    g = generator(rows, d_in, d_out)
    x = normal(g, rows, d_in, dtype=dtype, shift=shift)
    w = normal(g, d_out, d_in, dtype=dtype, scale=d_in ** -0.5, shift=shift)
    b = normal(g, d_out, dtype=dtype, scale=0.3, shift=shift) if bias else None
    r = normal(g, rows, d_out, dtype=dtype, shift=shift) if residual else None
    dy = normal(g, rows, d_out, dtype=dtype, shift=shift)
    y, z = lcn.lcn_linear(x, w, bias=b, residual=r, activation=ACTS[act], keep_pre=True)
    dx, dw, db = lcn.lcn_linear_backward(x, w, z, dy, activation=ACTS[act], with_bias=bias)
    ey, ez, edx, edw, edb = oracle(x, w, b, r, dy, act)
    assert off(z, ez) <= bound(F32, d_in)
    assert off(y, ey) <= bound(dtype, d_in)
    assert off(dx, edx) <= bound(dtype, d_out, 1)
    assert off(dw, edw) <= bound(dtype, rows, 1)
    assert (db is None) == (not bias)
    if bias:
        assert off(db, edb) <= bound(dtype, rows)
    return y, z, dx, dw, db


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [
    (1, 300, 20), (2, 64, 64), (7, 33, 5), (8, 128, 1), (9, 128, 1), (9, 1, 7), (40, 300, 32), (63, 72, 65), (257, 301, 130),
    (1000, 32, 32), (129, 2048, 257), (3000, 300, 512), (17, 4104, 12)])
def test_sizes(rows, d_in, d_out, dtype):
    check(rows, d_in, d_out, "tanh", dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("rows", [5, 300])
def test_activations(act, rows, dtype):
    check(rows, 96, 136, act, dtype)
    check(rows, 96, 136, act, dtype, bias=False, residual=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [3, 200])
def test_addresses_of_one_element(rows, dtype):
    check(rows, 64, 64, "gelu", dtype, shift=1)
    check(rows, 64, 62, "none", dtype, shift=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_tiles(dtype):
    check(5000, 512, 2050, "silu", dtype)


@pytest.mark.parametrize("rows,d_in,dtype", [(4103, 1024, BF16), (2053, 512, F32)])
def test_rows_behind_the_last_large_tile(rows, d_in, dtype):
    check(rows, d_in, 4096, "gelu", dtype)


def test_values_of_every_size_in_float():
    """Products of float values from 1e-18 to 1e18 are as exact as in single precision; the largest ones do not overflow."""
    g = generator(11)
    x, w = normal(g, 40, 64), normal(g, 48, 64)
    x = x * 10.0 ** torch.linspace(-18, 18, 40, device=DEV)[:, None]
    x[3, 5] = torch.finfo(F32).max
    w[:, 5] *= 1e-3
    y = lcn.lcn_linear(x, w)
    want = x.double() @ w.double().t().contiguous()
    for r in range(40):
        assert off(y[r], want[r]) <= bound(F32, 64)


def test_not_a_number_stays_in_its_row():
    g = generator(12)
    for dtype in (F32, BF16):
        for rows in (4, 100):
            x, w = normal(g, rows, 40, dtype=dtype), normal(g, 24, 40, dtype=dtype)
            x[2, 7] = math.nan
            y = lcn.lcn_linear(x, w, activation=lcn.ACT_RELU)
            assert torch.isnan(y[2]).all() and torch.isfinite(y[:2]).all() and torch.isfinite(y[3:]).all()


def test_same_bits_and_residual_in_place():
    g = generator(13)
    x, w, r = normal(g, 700, 300), normal(g, 300, 300), normal(g, 700, 300)
    a = lcn.lcn_linear(x, w, residual=r, activation=lcn.ACT_TANH)
    b = lcn.lcn_linear(x, w, residual=r, activation=lcn.ACT_TANH, out=r)
    assert b is r and torch.equal(a, b)
    dy = normal(g, 700, 300)
    first = lcn.lcn_linear_backward(x, w, None, dy)
    for u, v in zip(first, lcn.lcn_linear_backward(x, w, None, dy)):
        assert torch.equal(u, v)


def test_differences():
    """<dy, y> along a direction changes as the gradients say (central differences of the float path)."""
    g = generator(14)
    rows, d_in, d_out = 30, 20, 25
    x, w, b, dy = normal(g, rows, d_in), normal(g, d_out, d_in, scale=0.2), normal(g, d_out), normal(g, rows, d_out)
    for act in ("tanh", "gelu", "silu"):
        _, pre = lcn.lcn_linear(x, w, bias=b, activation=ACTS[act], keep_pre=True)
        grads = lcn.lcn_linear_backward(x, w, pre, dy, activation=ACTS[act])
        for at, grad in zip(range(3), grads):
            step = normal(g, *grad.shape)
            h = 1e-2 / step.norm().item() * math.sqrt(grad.numel()) * 0.1
            val = []
            for sign in (1, -1):
                args = [x, w, b]
                args[at] = args[at] + sign * h * step
                val.append((lcn.lcn_linear(args[0], args[1], bias=args[2], activation=ACTS[act]).double() * dy.double()).sum())
            want = (grad.double() * step.double()).sum().item()
            # the third derivative times h^2, and the rounding of the values over h
            room = 2e-4 * grad.double().norm().item() * step.double().norm().item()
            assert abs((val[0] - val[1]).item() / (2 * h) - want) <= room


def test_no_rows():
    w = torch.ones(5, 4, device=DEV)
    x = torch.empty(0, 4, device=DEV)
    assert lcn.lcn_linear(x, w).shape == (0, 5)
    dx, dw, db = lcn.lcn_linear_backward(x, w, None, torch.empty(0, 5, device=DEV))
    assert dx.shape == (0, 4) and not dw.any() and not db.any()


def test_other_stream_and_graph():
    g = generator(15)
    x, w, dy = normal(g, 600, 128, dtype=BF16), normal(g, 256, 128, dtype=BF16), normal(g, 600, 256, dtype=BF16)
    want = lcn.lcn_linear(x, w, activation=lcn.ACT_GELU, keep_pre=True)
    grads = lcn.lcn_linear_backward(x, w, want[1], dy, activation=lcn.ACT_GELU)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = lcn.lcn_linear(x, w, activation=lcn.ACT_GELU)
    side.synchronize()
    assert torch.equal(y, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lcn.lcn_linear(x, w, activation=lcn.ACT_GELU, keep_pre=True)
        gg = lcn.lcn_linear_backward(x, w, got[1], dy, activation=lcn.ACT_GELU)
    for _ in range(3):
        for t in (*got, *gg):
            t.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip((*got, *gg), (*want, *grads)):
            assert torch.equal(u, v)


def test_refusals():
    x, w = torch.ones(4, 6, device=DEV), torch.ones(3, 6, device=DEV)
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(x=x.bfloat16()), dict(w=torch.ones(3, 5, device=DEV)), dict(x=x.cpu()),
                dict(bias=torch.ones(4, device=DEV)), dict(residual=torch.ones(3, 4, device=DEV)),
                dict(bias=torch.ones(3, device=DEV, dtype=BF16)), dict(x=x[0])):
        args = dict(dict(x=x, w=w), **bad)
        with pytest.raises(ValueError):
            lcn.lcn_linear(**args)
    with pytest.raises(lcn.LcnError):
        lcn.lcn_linear(x, w, activation=9)
    with pytest.raises(lcn.LcnError):   # a workspace that is too small
        lcn.lcn_linear(torch.ones(99, 6, device=DEV), w, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(lcn.LcnError):   # an activation's gradient needs z
        lcn.lcn_linear_backward(x, w, None, torch.ones(4, 3, device=DEV), activation=lcn.ACT_TANH)


# ---- forms that the tests above leave out ------------------------------------------


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("rows,d_in,d_out", [(128, 8, 64), (300, 64, 200), (1000, 40, 33), (777, 128, 64), (515, 96, 20)])
def test_narrow_layers(rows, d_in, d_out, act, dtype):
    """Few inputs and outputs, rows of whole pieces: up to 32, 64 and 128 inputs, every activation."""
    check(rows, d_in, d_out, act, dtype)
    check(rows, d_in, d_out, act, dtype, bias=False, residual=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("rows,shift", [(5, 0), (300, 0), (700, 0), (300, 1)])
def test_single_gradients(rows, shift, act, dtype):
    """dx, dw and db have the same bits whichever are asked for."""
    g = generator(16, rows)
    x, w = normal(g, rows, 72, dtype=dtype, shift=shift), normal(g, 136, 72, dtype=dtype, shift=shift)
    dy, z = normal(g, rows, 136, dtype=dtype, shift=shift), normal(g, rows, 136)
    want = lcn.lcn_linear_backward(x, w, z, dy, activation=ACTS[act])
    for asked in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        got = lcn.lcn_linear_backward(x, w, z, dy, activation=ACTS[act], with_x=asked[0], with_w=asked[1], with_bias=asked[2])
        for a, u, v in zip(asked, got, want):
            assert torch.equal(u, v) if a else u is None

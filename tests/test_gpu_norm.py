"""lcn_layer_norm and lcn_layer_norm_backward against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, generator, normal, off, roundings

pytestmark = pytest.mark.gpu

EPS = 1e-5


def oracle(x, w, b, dy, around, eps=EPS):
    """y, mean, rstd, dx, dw, db in 64 bits, from the formulas."""
    x, dy = x.double(), dy.double()
    mean = x.mean(1, keepdim=True)
    rstd = 1.0 / ((x - mean).square().mean(1, keepdim=True) + eps).sqrt()
    xhat = (x - mean) * rstd
    y = xhat * (w.double() if w is not None else 1.0) + (b.double() if b is not None else 0.0)
    g = dy * (w.double() if w is not None else 1.0)
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if around is not None:
        dx = dx + around.double()
    return y, mean[:, 0], rstd[:, 0], dx, (dy * xhat).sum(0), dy.sum(0)


def inputs(rows, dim, dtype, shift=0, mean=0.5):
    g = generator(rows, dim)
    x = normal(g, rows, dim, dtype=dtype, shift=shift)
    x.add_(mean)
    w = normal(g, dim, dtype=dtype, scale=0.2, shift=shift)
    w.add_(1.0)
    return (x, w, normal(g, dim, dtype=dtype, scale=0.3, shift=shift), normal(g, rows, dim, dtype=dtype, shift=shift),
            normal(g, rows, dim, dtype=dtype, shift=shift))


def check(rows, dim, dtype, affine=True, around=True, shift=0):
    """Sums of `dim` or `rows` terms in 32 bits, results rounded once: no intermediate is rounded to bf16."""
    print("layer norm", rows, dim, dtype, affine, around, shift, flush=True)
    x, w, b, dy, a = inputs(rows, dim, dtype, shift)
    w, b, a = w if affine else None, b if affine else None, a if around else None
    y, mean, rstd = lcn.lcn_layer_norm(x, w, b, eps=EPS, keep_stats=True)
    assert torch.equal(y, lcn.lcn_layer_norm(x, w, b, eps=EPS))
    dx, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=a)
    want = oracle(x, w, b, dy, a)
    assert off(mean, want[1]) <= bound(F32, dim) and off(rstd, want[2]) <= bound(F32, dim)
    assert off(y, want[0]) <= bound(dtype, dim)
    # without a gradient around, narrow rows leave little of g when its two projections are taken out: the error is one of g
    room = 1.0 if around else max(1.0, (rstd.double()[:, None] * dy.double()).norm().item() / max(want[3].norm().item(), 1e-30))
    assert off(dx, want[3]) <= bound(F32, dim) * room + bound(dtype, dim)
    assert off(dw, want[4]) <= bound(dtype, rows + dim) and off(db, want[5]) <= bound(dtype, rows)
    return y, mean, rstd, dx, dw, db


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [
    (1, 16), (1, 2048), (2, 3), (5, 7), (3, 33), (64, 32), (1000, 32), (700, 40), (257, 63), (130, 64), (300, 100), (333, 129),
    (515, 300), (200, 301), (100, 512), (77, 1000), (64, 1024), (65, 1025), (50, 2048), (37, 2051), (33, 4096), (12, 8192),
    (7, 8193), (2100, 5281), (2053, 3333), (9, 8191), (9, 16384), (3, 20000), (2, 70001)])
def test_sizes(rows, dim, dtype):
    check(rows, dim, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(1, 64), (300, 24), (400, 300), (100, 2048), (20, 8200)])
def test_without_weights_or_a_gradient_around(rows, dim, dtype):
    check(rows, dim, dtype, affine=False)
    check(rows, dim, dtype, around=False)
    check(rows, dim, dtype, affine=False, around=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [32, 300, 1024, 4096])
def test_addresses_of_one_element(dim, dtype):
    check(90, dim, dtype, shift=1)
    check(90, dim, dtype, shift=4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(30000, 32), (20000, 300), (5000, 2048), (2048, 60), (2049, 129), (2200, 333), (2100, 350), (3001, 301),
                                      (2050, 1200), (2300, 200), (2111, 500), (2048, 4096)])
def test_many_rows(rows, dim, dtype):
    check(rows, dim, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(2100, 513), (300, 515), (2050, 767), (70, 1023), (2048, 2049), (40, 4099), (20, 8190), (9, 8195), (5, 16385)])
def test_long_rows_of_odd_widths(rows, dim, dtype):
    """Pieces of 16 bytes wherever they lie, of the last one only what exists; with what stands behind the last row left as it was."""
    check(rows, dim, dtype)
    y = check(rows, dim, dtype, shift=1)[0]
    x, w, b, _, _ = inputs(rows, dim, dtype, shift=1)
    room = torch.full((rows * dim + 64,), 7.0, dtype=dtype, device=DEV)
    assert torch.equal(lcn.lcn_layer_norm(x, w, b, eps=EPS, out=room[:rows * dim].view(rows, dim)), y)
    assert (room[rows * dim:] == 7.0).all()


def test_only_a_weight_or_only_a_bias():
    x, w, b, dy, _ = inputs(50, 96, F32)
    assert off(lcn.lcn_layer_norm(x, w), oracle(x, w, None, dy, None)[0]) <= bound(F32, 96)
    assert off(lcn.lcn_layer_norm(x, bias=b), oracle(x, None, b, dy, None)[0]) <= bound(F32, 96)


@pytest.mark.parametrize("dim", [32, 300, 4096, 9000])
def test_a_mean_far_from_zero(dim):
    """Differences to the mean, no difference of squares: with a mean of 1000 deviations the values' own spacing is what is left.
    The mean is off by sqrt(dim) halves of 2^-24 of itself at most, and so is x - mean."""
    x, w, b, dy, around = inputs(40, dim, F32, mean=1000.0)
    y, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    want = oracle(x, w, b, dy, around)
    room = 1000.0 * 2.0 ** -24 * (2 + math.sqrt(dim) / 8) + bound(F32, dim)
    assert off(y, want[0]) <= room and off(rstd, want[2]) <= room


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_equal_values(dtype):
    """No variance: y is the bias, whatever the value is, and dx is g less its mean over sqrt(eps)."""
    g = generator(3)
    for dim in (32, 300, 8200):
        x = torch.full((5, dim), 3.0, dtype=dtype, device=DEV)
        w, b, dy = normal(g, dim, dtype=dtype), normal(g, dim, dtype=dtype), normal(g, 5, dim, dtype=dtype)
        y, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
        assert torch.equal(y, b.expand(5, dim))
        dx, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy)
        assert not dw.any()
        assert off(dx, oracle(x, w, b, dy, None)[3]) <= bound(dtype, dim)
        assert torch.isnan(lcn.lcn_layer_norm(x, w, b, eps=0.0)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [24, 300, 2048, 9000])
def test_what_is_not_finite_stays_in_its_row(dim, dtype):
    x, w, b, dy, _ = inputs(70, dim, dtype)
    want = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    x[3, 5], x[40, 0], x[69, dim - 1] = math.nan, math.inf, -math.inf
    y, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    bad = torch.tensor([3, 40, 69], device=DEV)
    fine = torch.tensor([r for r in range(70) if r not in (3, 40, 69)], device=DEV)
    assert torch.isnan(y[bad]).all()
    for u, v in zip((y, mean, rstd), want):
        assert torch.equal(u[fine], v[fine])
    dx, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[fine]).all() and torch.isfinite(db).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(300, 32), (100, 300), (60, 4096), (5, 9000)])
def test_single_gradients_and_same_bits(rows, dim, dtype):
    """dx, dw and db have the same bits whichever are asked for, and from call to call."""
    x, w, b, dy, around = inputs(rows, dim, dtype)
    _, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    want = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=around)
    for asked in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        got = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=around, with_x=asked[0], with_weight=asked[1],
                                          with_bias=asked[2])
        for a, u, v in zip(asked, got, want):
            assert torch.equal(u, v) if a else u is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [32, 300, 301, 4096, 9000])
def test_in_place(dim, dtype):
    x, w, b, _, _ = inputs(45, dim, dtype)
    want = lcn.lcn_layer_norm(x, w, b)
    assert lcn.lcn_layer_norm(x, w, b, out=x) is x and torch.equal(x, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(45, 32), (2100, 300), (45, 301), (3000, 2048), (33, 9000)])
def test_dx_in_place_of_the_gradient_around(rows, dim, dtype):
    """dx may be the memory of `around` (the C entry point; the binding's dx is new)."""
    from paper_2107_06876_amd import encoder
    x, w, b, dy, around = inputs(rows, dim, dtype)
    _, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    want, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=around)
    sizes = (rows, dim, 0 if dtype == F32 else 1)
    space = torch.empty(encoder._bytes("lcn_layer_norm_workspace_bytes", sizes), dtype=torch.uint8, device=DEV)
    got = torch.empty(2, dim, dtype=dtype, device=DEV)
    encoder._call("lcn_layer_norm_backward", x.device, x.data_ptr(), w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dy.data_ptr(),
                  around.data_ptr(), *sizes, around.data_ptr(), got[0].data_ptr(), got[1].data_ptr(), space.data_ptr(), space.numel())
    assert torch.equal(around, want) and torch.equal(got[0], dw) and torch.equal(got[1], db)


def test_values_of_every_size():
    """A row's size drops out, up to eps on one side and the range of squares on the other."""
    x, w, b, _, _ = inputs(40, 300, F32)
    want = lcn.lcn_layer_norm(x, w, b, eps=0.0)
    for size in (1e-15, 1e-6, 1e6, 1e18):
        assert off(lcn.lcn_layer_norm(x * size, w, b, eps=0.0), want) <= 4 * bound(F32, 300)
    assert off(lcn.lcn_layer_norm(x * 1e25, w, b), b.expand(40, 300)) == 0.0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(5, 16), (70, 300), (2050, 300), (9, 301), (2100, 513), (33, 4096), (2048, 4096), (5, 9000), (3, 20001)])
def test_rows_up_to_the_largest_values(rows, dim, dtype):
    """Sums and differences of finite rows leave a float's range where the mean and the variance do, not before: y is the bias, the mean
    is off by the roundings of its sum, and what reaches x is the gradient around."""
    g = generator(rows, dim)
    w, b, dy, around = (normal(g, *shape, dtype=dtype) for shape in ((dim,), (dim,), (rows, dim), (rows, dim)))
    sign = torch.randint(0, 2, (rows, dim), generator=g).to(DEV) * 2.0 - 1.0
    one = torch.ones(rows, dim, device=DEV)
    one[:, dim // 2] = -1.0
    for x in (sign * 1e36, sign * 3.3e38, one * 3.3e38, one.abs() * 1e36, one.abs() * 3.3e38, one.abs() * -3.3e38):
        x = x.to(dtype)
        assert torch.isfinite(x).all()
        y, mean, rstd = lcn.lcn_layer_norm(x, w, b, eps=EPS, keep_stats=True)
        assert torch.equal(y, b.expand(rows, dim))
        largest = x.double().abs().amax(1)
        assert ((mean.double() - x.double().mean(1)).abs() <= largest * (dim * 2.0 ** -24)).all()
        if (x[0] != x[0, 0]).any():
            assert not rstd.any()
            dx, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=around)
            assert torch.equal(dx, around) and not dw.any() and off(db, dy.double().sum(0)) <= bound(dtype, rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,dim", [(3, 2), (70, 6), (2050, 24), (70, 300), (2050, 300), (9, 302), (2100, 514), (33, 1000), (5, 3002), (5, 9000),
                                      (3, 20002)])
def test_a_variance_of_one(rows, dim, dtype):
    """Rows of 1 and -1: every sum is exact, and so are the variance, rstd and y."""
    x = torch.ones(rows, dim, dtype=dtype, device=DEV)
    x[:, ::2] = -1.0
    y, mean, rstd = lcn.lcn_layer_norm(x, eps=0.0, keep_stats=True)
    assert torch.equal(y, x) and not mean.any() and (rstd == 1.0).all()


@pytest.mark.parametrize("dim", [64, 300, 4096])
def test_roundings_of_bf16(dim):
    x, w, b, dy, around = inputs(2000, dim, BF16)
    y, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    got = (y, *lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=around))
    want = oracle(x, w, b, dy, around)
    for u, v in zip(got, (want[0], *want[3:])):
        assert off(u, v) <= roundings(1)


@pytest.mark.parametrize("rows,dim", [(40961, 300), (30000, 1024), (8000, 4096)])
def test_sums_over_rows_in_pairs(rows, dim):
    """Sums of random terms: a sum in pairs adds one rounding's square to the error's with every doubling, a chain of m sums m / 2 of them.
    Up to 512 workgroups have rows / 512 of them, in chains of up to 16 and then in pairs; their sums are added in
    chains of 8, then in pairs: 6 doublings.  A rounding is 0.737 2^-23 / sqrt(12) in the 2-norm, and 1.15 leaves room for what it varies by."""
    x, w, b, dy, _ = inputs(rows, dim, F32)
    y, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    _, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, with_x=False)
    chain = {300: 5, 1024: 15, 4096: 16}[dim] / 2   # of a thread's rows
    pairs = {300: 4, 1024: 2, 4096: 0}[dim]         # lanes and wavefronts of a workgroup that share columns
    doublings = chain + pairs + 4 + 6
    assert off(db, dy.double().sum(0)) <= 1.15 * 0.737 * 2.0 ** -23 / math.sqrt(12.0) * math.sqrt(doublings)


def test_differences():
    """<dy, y> changes along a direction as the gradients say (central differences of the float path)."""
    g = generator(5)
    x, w, b, dy, _ = inputs(30, 40, F32)
    _, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
    grads = lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy)
    for at, grad in enumerate(grads):
        step = normal(g, *grad.shape)
        h = 1e-2
        val = []
        for sign in (1, -1):
            args = [x, w, b]
            args[at] = args[at] + sign * h * step
            val.append((lcn.lcn_layer_norm(*args).double() * dy.double()).sum().item())
        # h^2 / 6 of the third derivative (a few times rstd^3 |dy| |step|^3 / sqrt(dim)) and the values' rounding over h
        room = 1e-3 * grad.double().norm().item() * step.double().norm().item()
        assert abs((val[0] - val[1]) / (2 * h) - (grad.double() * step.double()).sum().item()) <= room


def test_no_rows():
    x, w = torch.empty(0, 12, device=DEV), torch.ones(12, device=DEV)
    y, mean, rstd = lcn.lcn_layer_norm(x, w, keep_stats=True)
    assert y.shape == (0, 12) and mean.shape == (0,)
    dx, dw, db = lcn.lcn_layer_norm_backward(x, w, mean, rstd, x)
    assert dx.shape == (0, 12) and not dw.any() and not db.any()


@pytest.mark.parametrize("rows,dim", [(500, 32), (300, 300), (120, 2048), (3, 9000)])
def test_other_stream_and_graph(rows, dim):
    x, w, b, dy, around = inputs(rows, dim, BF16)

    def both():
        y, mean, rstd = lcn.lcn_layer_norm(x, w, b, keep_stats=True)
        return (y, mean, rstd, *lcn.lcn_layer_norm_backward(x, w, mean, rstd, dy, around=around))

    want = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    for u, v in zip(got, want):
        assert torch.equal(u, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        for t in got:
            t.fill_(-7.0)
        both()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, want):
            assert torch.equal(u, v)


def test_refusals():
    x, w = torch.ones(4, 6, device=DEV), torch.ones(6, device=DEV)
    s = torch.ones(4, device=DEV)
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(x=x.bfloat16()), dict(weight=w[:5]), dict(x=x.cpu()), dict(x=x[0]),
                dict(bias=w.bfloat16()), dict(out=torch.ones(4, 5, device=DEV)), dict(x=torch.ones(4, 0, device=DEV))):
        with pytest.raises(ValueError):
            lcn.lcn_layer_norm(**dict(dict(x=x, weight=w), **bad))
    for eps in (-1.0, math.nan, math.inf):
        with pytest.raises(lcn.LcnError):
            lcn.lcn_layer_norm(x, w, eps=eps)
    good = dict(x=x, weight=w, mean=s, rstd=s, dy=x)
    for bad in (dict(mean=s[:3]), dict(rstd=s.bfloat16()), dict(dy=x[:3]), dict(dy=x.t()), dict(around=x[:2]), dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            lcn.lcn_layer_norm_backward(**dict(good, **bad))
    for bad in (dict(mean=None), dict(rstd=None), dict(dy=None), dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises(lcn.LcnError):
            lcn.lcn_layer_norm_backward(**dict(good, **bad))

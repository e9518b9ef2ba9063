"""lcn_orthogonalise against the same products in 64 bits, and against a decomposition."""
import math

import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, generator, normal, off, roundings

pytestmark = pytest.mark.gpu

UPDATE, MAP = lcn.ORTHOGONAL_UPDATE, lcn.ORTHOGONAL_MAP
EPS = 1e-7


def triples(steps, coefficients):
    return [coefficients] * steps if isinstance(coefficients[0], float) else list(coefficients)


def oracle(g, steps, coefficients, eps=EPS):
    """X of one matrix in 64 bits, and how far 32-bit products may take it.

    What a step's three products and the rounding of its planes add is at most bound(F32, k) of the factors' sizes, |X_k| times the
    largest of a + b t + c t^2 over the spectrum (for B X, and for B the same again twice).  The steps behind it let that grow by the
    polynomial's largest slope each, which is a at 0 for the coefficients here (up to their own values beyond it)."""
    x = g.double().cpu()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    x = x / (x.norm() + eps)
    error = 0.0
    for a, b, c in triples(steps, coefficients):
        gram = x @ x.t()
        slope = max(abs(a + 3 * b * t + 5 * c * t * t) for t in [i / 64 * 1.5 for i in range(65)])
        most = max(abs(a + b * t + c * t * t) for t in [i / 64 * 1.5 for i in range(65)])
        error = error * slope + 3 * bound(F32, x.shape[1]) * most * x.norm().item()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.t() if tall else x).to(DEV), error / x.norm().item()


def gradient(key, rows, cols, dtype=F32, shift=0):
    """A product of samples, as gradients of weights are."""
    g = generator(key, rows, cols)
    k = 2 * min(rows, cols)
    m = torch.randn(rows, k, generator=g) @ (torch.randn(k, cols, generator=g) * torch.arange(1, cols + 1) ** -0.25) * (0.01 / k)
    flat = torch.zeros(rows * cols + shift, dtype=dtype, device=DEV)
    flat[shift:] = m.to(dtype).to(DEV).flatten()
    return flat[shift:].view(rows, cols)


def check(rows, cols, dtype, steps=5, coefficients=UPDATE, shift=0):
    print("orthogonalise", rows, cols, dtype, steps, coefficients, shift, flush=True)
    g = gradient(1, rows, cols, dtype, shift)
    x = lcn.lcn_orthogonalise(g, steps=steps, coefficients=coefficients, eps=EPS)
    want, room = oracle(g, steps, coefficients)
    print("  off", off(x, want), "room", room, flush=True)
    assert off(x, want) <= room + (2.0 ** -8 if dtype == BF16 else 0.0)
    return x


SIZES = [(1, 1), (1, 7), (9, 1), (2, 3), (16, 16), (31, 33), (32, 96), (96, 32), (64, 64), (65, 64), (40, 200), (200, 40), (129, 127),
         (300, 300), (1024, 300), (300, 1024), (257, 513), (512, 512), (700, 701), (1031, 1030)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, dtype):
    check(rows, cols, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(8, 3000), (5000, 24), (64, 10000), (2000, 500), (520, 4097)])
def test_long_matrices(rows, cols, dtype):
    check(rows, cols, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(640, 640), (621, 707), (100, 4000), (35, 600), (5001, 161), (300, 300), (900, 890), (33, 1037)])
def test_small_tiles(rows, cols, dtype):
    """Few tiles: all of a symmetric product, its half written twice, sums split over workgroups."""
    check(rows, cols, dtype)


@pytest.mark.parametrize("rows,cols", [(2048, 2304), (2311, 1100)])
def test_large_tiles(rows, cols):
    check(rows, cols, BF16, steps=3)
    check(rows, cols, F32, steps=2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(20, 50), (64, 64), (300, 128), (100, 333)])
def test_addresses_of_one_element(rows, cols, dtype):
    check(rows, cols, dtype, shift=1)
    check(rows, cols, dtype, shift=4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("steps", [1, 2, 3, 7, 12])
def test_steps_and_coefficients(steps, dtype):
    for rows, cols in ((48, 80), (150, 150), (400, 200)):
        check(rows, cols, dtype, steps=steps)
        check(rows, cols, dtype, steps=steps, coefficients=MAP)
        check(rows, cols, dtype, steps=steps, coefficients=[UPDATE if i % 2 else MAP for i in range(steps)])
        check(rows, cols, dtype, steps=steps, coefficients=(1.5, -0.5, 0.0))


@pytest.mark.parametrize("rows,cols", [(30, 30), (60, 90), (200, 120)])
def test_the_nearest_orthogonal_map(rows, cols):
    """Singular values from 1 down to 1/20 go to 1: the polar factor U V^T of a decomposition."""
    g = generator(7, rows, cols)
    lo = min(rows, cols)
    u, _ = torch.linalg.qr(torch.randn(rows, lo, generator=g, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(cols, lo, generator=g, dtype=torch.float64))
    m = ((u * torch.linspace(1.0, 0.05, lo, dtype=torch.float64)) @ v.t()).float().to(DEV)
    # the norm is sqrt(lo) at most, so that the smallest value starts above 0.05 / sqrt(200) and grows by 1.875 a step: 15 steps
    x = lcn.lcn_orthogonalise(m, steps=18, coefficients=MAP)
    # in rounding m to float its singular vectors move by 2^-24 |m| over their gap to the others' negative, 0.1
    assert off(x, (u @ v.t()).to(DEV)) <= 2.0 ** -24 * math.sqrt(lo) * 20 + 3 * bound(F32, max(rows, cols))
    one = x.t() @ x if rows >= cols else x @ x.t()
    assert off(one, torch.eye(lo, device=DEV)) <= 8 * bound(F32, max(rows, cols))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("count,rows,cols", [(8, 96, 32), (3, 20, 70), (2, 300, 200), (5, 130, 257), (70, 5, 9), (3, 512, 1024)])
def test_batches(count, rows, cols, dtype):
    g = torch.stack([gradient(i, rows, cols, dtype) * 10.0 ** (i % 7 - 3) for i in range(count)])
    g[count // 2] = 0.0
    x = lcn.lcn_orthogonalise(g)
    assert x.shape == g.shape and not x[count // 2].any()
    for i in range(count):
        if i != count // 2:
            want, room = oracle(g[i], 5, UPDATE)
            assert off(x[i], want) <= room + (2.0 ** -8 if dtype == BF16 else 0.0)


@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 500), (900, 600), (1500, 1024), (100, 800), (1200, 128), (4100, 520)])
def test_one_rounding_of_bf16(rows, cols):
    g = gradient(3, rows, cols, BF16)
    assert off(lcn.lcn_orthogonalise(g), oracle(g, 5, UPDATE)[0]) <= roundings(1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(96, 60), (400, 300), (900, 100)])
def test_few_directions(rows, cols, dtype):
    """A gradient of 6 samples has 6 singular values beside those of its rounding, which grow the most: also they come out."""
    g = generator(9, rows, cols)
    m = (torch.randn(rows, 6, generator=g) @ torch.randn(6, cols, generator=g) * 1e-3).to(dtype).to(DEV)
    want, room = oracle(m, 5, UPDATE)
    x = lcn.lcn_orthogonalise(m)
    assert off(x, want) <= room + (2.0 ** -8 if dtype == BF16 else 0.0)


def test_sizes_of_every_order_in_float():
    """The norm is formed in 64 bits: squares may leave a float's range."""
    base = gradient(4, 40, 60)
    base = base / base.norm()
    want = lcn.lcn_orthogonalise(base, eps=0.0)
    for size in (1e-37, 1e-30, 1e-20, 1e20, 1e30, 1e37):
        assert off(lcn.lcn_orthogonalise(base * size, eps=0.0), want) <= 1e-4
    assert off(lcn.lcn_orthogonalise(base * 1e-7), oracle(base * 1e-7, 5, UPDATE)[0]) <= oracle(base * 1e-7, 5, UPDATE)[1]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(40, 24), (150, 200)])
def test_what_is_not_finite_stays_in_its_matrix(rows, cols, dtype):
    g = torch.stack([gradient(i, rows, cols, dtype) for i in range(4)])
    want = lcn.lcn_orthogonalise(g)
    g[1, 3, 5], g[3, rows - 1, cols - 1] = math.nan, math.inf
    x = lcn.lcn_orthogonalise(g)
    assert torch.isnan(x[1]).all() and torch.isnan(x[3]).all()
    assert torch.equal(x[0], want[0]) and torch.equal(x[2], want[2])
    assert torch.isnan(lcn.lcn_orthogonalise(torch.zeros(rows, cols, dtype=dtype, device=DEV), eps=0.0)).all()
    assert not lcn.lcn_orthogonalise(torch.zeros(rows, cols, dtype=dtype, device=DEV)).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(96, 32), (300, 301)])
def test_in_place_scaled_and_same_bits(rows, cols, dtype):
    g = torch.stack([gradient(i, rows, cols, dtype) for i in range(2)])
    want = lcn.lcn_orthogonalise(g)
    assert torch.equal(want, lcn.lcn_orthogonalise(g))
    assert off(lcn.lcn_orthogonalise(g, scale=-0.25), -0.25 * want) == 0.0   # a power of two is exact
    assert lcn.lcn_orthogonalise(g, out=g) is g and torch.equal(g, want)


# ---- long bf16 matrices, whose steps are taken on A alone, several to a stage ----


@pytest.mark.parametrize("steps", [1, 2, 3, 6, 7, 12, 13])
@pytest.mark.parametrize("rows,cols", [(900, 100), (100, 800), (70, 1030)])
def test_steps_and_coefficients_of_long_matrices(rows, cols, steps):
    check(rows, cols, BF16, steps=steps)
    check(rows, cols, BF16, steps=steps, coefficients=MAP)
    check(rows, cols, BF16, steps=steps, coefficients=[UPDATE if i % 2 else MAP for i in range(steps)])
    check(rows, cols, BF16, steps=steps, coefficients=[MAP if i % 3 else UPDATE for i in range(steps)])
    check(rows, cols, BF16, steps=steps, coefficients=(1.5, -0.5, 0.0))


@pytest.mark.parametrize("count,rows,cols", [(4, 900, 100), (3, 100, 800), (5, 1200, 128), (3, 65, 500), (3, 2500, 600)])
def test_batches_of_long_matrices(count, rows, cols):
    """Matrices of different sizes each have their own factor; one of zeros stays so, also beside others."""
    g = torch.stack([gradient(i, rows, cols, BF16) * 10.0 ** (3 * i - 6) for i in range(count)])
    g[count // 2] = 0.0
    for steps, coefficients in ((5, UPDATE), (9, MAP)):
        x = lcn.lcn_orthogonalise(g, steps=steps, coefficients=coefficients)
        assert not x[count // 2].any()
        for i in range(count):
            if i != count // 2:
                want, room = oracle(g[i], steps, coefficients)
                assert off(x[i], want) <= room + 2.0 ** -8


@pytest.mark.parametrize("rows,cols", [(900, 100), (100, 800)])
def test_what_is_not_finite_stays_in_its_long_matrix(rows, cols):
    g = torch.stack([gradient(i, rows, cols, BF16) for i in range(5)])
    for steps, coefficients in ((5, UPDATE), (1, UPDATE), (6, MAP)):
        want = lcn.lcn_orthogonalise(g, steps=steps, coefficients=coefficients)
        bad = g.clone()
        bad[1, 3, 5], bad[2, 0, 0], bad[4, rows - 1, cols - 1] = math.nan, -math.inf, math.inf
        x = lcn.lcn_orthogonalise(bad, steps=steps, coefficients=coefficients)
        for i in range(5):
            assert torch.isnan(x[i]).all() if i in (1, 2, 4) else torch.equal(x[i], want[i])
    zero = torch.zeros(2, rows, cols, dtype=BF16, device=DEV)
    assert torch.isnan(lcn.lcn_orthogonalise(zero, eps=0.0)).all() and not lcn.lcn_orthogonalise(zero).any()


@pytest.mark.parametrize("rows,cols", [(900, 100), (100, 800), (4100, 520)])
def test_long_matrices_in_place_scaled_and_same_bits(rows, cols):
    g = torch.stack([gradient(i, rows, cols, BF16) for i in range(3)])
    want = lcn.lcn_orthogonalise(g, steps=7, coefficients=MAP)
    assert torch.equal(want, lcn.lcn_orthogonalise(g, steps=7, coefficients=MAP))
    for i in range(3):   # and of each alone
        assert off(lcn.lcn_orthogonalise(g[i], steps=7, coefficients=MAP), want[i].double()) <= 2.0 ** -8
    assert off(lcn.lcn_orthogonalise(g, steps=7, coefficients=MAP, scale=-0.25), -0.25 * want) == 0.0
    assert lcn.lcn_orthogonalise(g, steps=7, coefficients=MAP, out=g) is g and torch.equal(g, want)


@pytest.mark.parametrize("rows,cols", [(900, 100), (100, 800)])
def test_sizes_of_every_order_of_long_matrices(rows, cols):
    """bf16 has a float's range: the factor of a matrix is a power of two and the rest.  (The least values, 2^-31, lose bits as
    subnormals at 2^-100: what is compared with is the matrix that is left.)"""
    base = gradient(4, rows, cols, BF16)
    for power in (-100, -60, 60, 120):
        g = base * 2.0 ** power
        left = (g.double() * 2.0 ** -power).bfloat16()
        assert torch.equal(left.double() * 2.0 ** power, g.double())
        assert torch.equal(lcn.lcn_orthogonalise(g, eps=0.0), lcn.lcn_orthogonalise(left, eps=0.0))


def test_no_matrices():
    assert lcn.lcn_orthogonalise(torch.empty(0, 4, 5, device=DEV)).shape == (0, 4, 5)


@pytest.mark.parametrize("count,rows,cols", [(8, 96, 32), (1, 300, 300), (2, 700, 400)])
def test_other_stream_and_graph(count, rows, cols):
    g = torch.stack([gradient(i, rows, cols, BF16) for i in range(count)])
    want = lcn.lcn_orthogonalise(g)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = lcn.lcn_orthogonalise(g)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lcn.lcn_orthogonalise(g)
    other = g * 2.0 + 0.01
    for source in (g, other, g):
        keep = g.clone()
        g.copy_(source)
        want = lcn.lcn_orthogonalise(g)
        got.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        g.copy_(keep)


def test_refusals():
    g = torch.ones(4, 6, device=DEV)
    for bad in (g.t(), g.half(), g.cpu(), g[0], g[None, None], torch.ones(4, 0, device=DEV)):
        with pytest.raises(ValueError):
            lcn.lcn_orthogonalise(bad)
    for bad in (dict(steps=0), dict(coefficients=(1.0, 2.0)), dict(coefficients=[UPDATE] * 4), dict(out=torch.ones(6, 4, device=DEV)),
                dict(out=g.bfloat16())):
        with pytest.raises(ValueError):
            lcn.lcn_orthogonalise(g, **bad)
    for bad in (dict(steps=65), dict(eps=-1.0), dict(eps=math.nan), dict(scale=math.inf), dict(coefficients=(math.nan, 0.0, 0.0)),
                dict(coefficients=(5.0, 0.0, 0.0)), dict(coefficients=(100.0, -300.0, 200.0))):
        with pytest.raises(lcn.LcnError):
            lcn.lcn_orthogonalise(g, **bad)
    with pytest.raises(lcn.LcnError):   # a workspace that is too small
        lcn.lcn_orthogonalise(torch.ones(300, 300, device=DEV), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))

"""lcn_gated_linear and lcn_gated_linear_backward against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, farthest, generator, normal, off, roundings

pytestmark = pytest.mark.gpu

ACTS = {"none": lcn.ACT_NONE, "tanh": lcn.ACT_TANH, "relu": lcn.ACT_RELU, "gelu": lcn.ACT_GELU, "silu": lcn.ACT_SILU}
FUNCTIONS = dict(none=lambda z: z * 1.0, tanh=torch.tanh, relu=torch.relu, gelu=torch.nn.functional.gelu,
                 silu=torch.nn.functional.silu)


def oracle(x, w, b, dy, act):
    """y, [g | u], dx, dw, db in 64 bits."""
    x, w, dy = x.double(), w.double(), dy.double()
    d = w.shape[0] // 2
    z = x @ w.t().contiguous()
    if b is not None:
        z = z + b.double()
    z = z.detach().requires_grad_(True)
    y = FUNCTIONS[act](z[:, :d]) * z[:, d:]
    (dz,) = torch.autograd.grad(y, z, dy)
    return y.detach(), z.detach(), dz @ w, dz.t().contiguous() @ x, dz.sum(0)


def inputs(rows, d_in, d_out, dtype, shift=0):
    g = generator(rows, d_in, d_out)
    return (normal(g, rows, d_in, dtype=dtype, shift=shift), normal(g, 2 * d_out, d_in, dtype=dtype, scale=d_in ** -0.5, shift=shift),
            normal(g, 2 * d_out, dtype=dtype, scale=0.3, shift=shift), normal(g, rows, d_out, dtype=dtype, shift=shift))


def check(rows, d_in, d_out, act, dtype, bias=True, shift=0):
    """g and u are off by the error of a sum of d_in terms each, y by both and (through act) once more; dz as y, rounded to bf16 on
    its way into the products."""
    print("gated", rows, d_in, d_out, act, dtype, bias, shift, flush=True)
    x, w, b, dy = inputs(rows, d_in, d_out, dtype, shift)
    b = b if bias else None
    y, z = lcn.lcn_gated_linear(x, w, bias=b, activation=ACTS[act], keep_pre=True)
    assert torch.equal(y, lcn.lcn_gated_linear(x, w, bias=b, activation=ACTS[act]))
    dx, dw, db = lcn.lcn_gated_linear_backward(x, w, z, dy, activation=ACTS[act], with_bias=bias)
    ey, ez, edx, edw, edb = oracle(x, w, b, dy, act)
    own = 3 * bound(F32, d_in)
    y_room = own + bound(dtype, 1)
    if dtype == BF16:   # g and u are kept within 2^-14 of the power of two above the largest of eight, less than 4 of their norm's share
        own += 2 * 2.0 ** -14 * 4
    if act == "relu":   # its slope jumps: a g within the rounding of 0 may have either slope (it has one in expectation 1e-6 of places)
        near = (ez[:, :d_out].abs() <= (2.0 ** -20 if dtype == F32 else 2.0 ** -11)).sum().item()
        own += math.sqrt(near / ez[:, :d_out].numel())
    assert off(y, ey) <= y_room
    assert off(dx, edx) <= own + bound(dtype, 2 * d_out, 1)
    assert off(dw, edw) <= own + bound(dtype, rows, 1)
    assert (db is None) == (not bias)
    if bias:
        assert off(db, edb) <= own + bound(dtype, rows)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [
    (1, 300, 20), (1, 1, 1), (2, 64, 64), (3, 17, 129), (7, 33, 5), (8, 128, 1), (9, 128, 1), (9, 1, 7), (40, 300, 32), (63, 72, 65),
    (64, 64, 32), (257, 301, 130), (1000, 32, 64), (129, 2048, 257), (3000, 300, 512), (17, 4104, 12), (100, 40, 31), (65, 48, 100),
    (700, 56, 33), (515, 96, 20), (300, 64, 200), (130, 1000, 66)])
def test_sizes(rows, d_in, d_out, dtype):
    check(rows, d_in, d_out, "silu", dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("rows,d_in,d_out", [(5, 96, 136), (300, 96, 136), (777, 32, 64)])
def test_activations(act, rows, d_in, d_out, dtype):
    check(rows, d_in, d_out, act, dtype)
    check(rows, d_in, d_out, act, dtype, bias=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [3, 200])
def test_addresses_of_one_element(rows, dtype):
    check(rows, 64, 64, "gelu", dtype, shift=1)
    check(rows, 64, 62, "none", dtype, shift=1)
    check(rows, 64, 64, "silu", dtype, shift=4)


@pytest.mark.parametrize("rows,d_in,d_out,dtype", [(5000, 512, 1026, BF16), (4103, 1024, 2048, BF16), (2053, 512, 2048, F32),
                                                   (3000, 200, 1025, F32)])
def test_large_tiles(rows, d_in, d_out, dtype):
    check(rows, d_in, d_out, "silu", dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("rows,d_in,d_out", [(128, 8, 64), (300, 64, 40), (1000, 40, 33), (777, 32, 64), (515, 56, 20), (129, 16, 1),
                                             (4099, 64, 64), (20000, 32, 31)])
def test_narrow_layers(rows, d_in, d_out, act, dtype):
    """Few inputs and outputs: up to 32 and 64 of either, every activation; dz is not rounded there."""
    check(rows, d_in, d_out, act, dtype)
    check(rows, d_in, d_out, act, dtype, bias=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [(300, 33, 64), (5000, 61, 50), (129, 1, 3), (128, 63, 1), (4097, 31, 63), (200, 30, 7)])
def test_narrow_layers_of_odd_widths(rows, d_in, d_out, dtype):
    """Rows that are no whole pieces, from addresses that are none either."""
    check(rows, d_in, d_out, "silu", dtype)
    check(rows, d_in, d_out, "tanh", dtype, bias=False, shift=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [(1, 2047, 333), (2, 1025, 100), (4, 519, 61), (8, 2051, 77), (3, 7, 9), (1, 129, 16)])
def test_few_rows_of_odd_widths(rows, d_in, d_out, dtype):
    check(rows, d_in, d_out, "silu", dtype)
    check(rows, d_in, d_out, "gelu", dtype, shift=1)


@pytest.mark.parametrize("rows", [9, 16, 17, 31, 32, 33, 48, 49, 64, 65])
@pytest.mark.parametrize("d_in,d_out", [(1, 1), (33, 17), (96, 136), (301, 15), (130, 1025), (1024, 16), (1025, 40)])
def test_some_rows(rows, d_in, d_out):
    """Tiles of 16 rows and outputs that are not full, k that four wavefronts share unevenly or not at all."""
    check(rows, d_in, d_out, "silu", F32)
    check(rows, d_in, d_out, "gelu", F32, bias=False, shift=1)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_activations_of_some_rows(act, dtype):
    check(20, 100, 50, act, dtype)
    check(12, 2056, 24, act, dtype, bias=False)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [(300, 32, 64), (1000, 64, 33)])
def test_single_gradients_of_narrow_layers(rows, d_in, d_out, dtype):
    x, w, b, dy = inputs(rows, d_in, d_out, dtype)
    _, z = lcn.lcn_gated_linear(x, w, bias=b, keep_pre=True)
    want = lcn.lcn_gated_linear_backward(x, w, z, dy)
    for asked in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        got = lcn.lcn_gated_linear_backward(x, w, z, dy, with_x=asked[0], with_w=asked[1], with_bias=asked[2])
        for a, u, v in zip(asked, got, want):
            assert torch.equal(u, v) if a else u is None


@pytest.mark.parametrize("rows", [12, 300, 512, 700, 4103])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_roundings_of_bf16(act, rows):
    """y and db are rounded once; dz is rounded as well on its way into dx and dw, above 512 rows."""
    d_in, d_out = (264, 520) if rows < 4000 else (512, 2048)
    x, w, b, dy = inputs(rows, d_in, d_out, BF16)
    y, z = lcn.lcn_gated_linear(x, w, bias=b, activation=ACTS[act], keep_pre=True)
    got = (y, *lcn.lcn_gated_linear_backward(x, w, z, dy, activation=ACTS[act]))
    want = oracle(x, w, b, dy, act)
    once = 1 if rows <= 512 else 2
    # y and dz are products of values with many sizes, spread more evenly over octaves: 1.1 covers that
    for u, v, n in zip(got, (want[0], *want[2:]), (1, once, once, 1)):
        assert off(u, v) <= roundings(n) and farthest(u, v) <= 1.0


def test_not_a_number_stays_in_its_row():
    for dtype in (F32, BF16):
        for rows in (4, 100, 300):
            x, w, b, _ = inputs(rows, 40, 24, dtype)
            x[2, 7] = math.nan
            y = lcn.lcn_gated_linear(x, w, bias=b, activation=lcn.ACT_SILU)
            assert torch.isnan(y[2]).all() and torch.isfinite(y[:2]).all() and torch.isfinite(y[3:]).all()
            x, w, b, _ = inputs(rows, 40, 24, dtype)
            w[24 + 5, 3] = math.nan   # a row of Wu: one output
            y = lcn.lcn_gated_linear(x, w, bias=b, activation=lcn.ACT_SILU)
            assert torch.isnan(y[:, 5]).all() and torch.isfinite(y[:, :5]).all() and torch.isfinite(y[:, 6:]).all()


@pytest.mark.parametrize("rows,d_out", [(3, 40), (3, 37), (100, 64), (300, 37), (700, 520)])
def test_what_is_kept_has_any_size(rows, d_out):
    """g and u of bf16 tensors are kept with an exponent for eight: the gradients of layers with values from 1e-18 to 1e18, and in
    one layer of columns from 1e-6 to 1e6, are as exact as those of values near 1."""
    x, w, _, dy = inputs(rows, 48, d_out, BF16)
    for sizes in (1e-18, 1e18, 10.0 ** torch.linspace(-6, 6, d_out, device=DEV)):
        s = torch.as_tensor(sizes, device=DEV).expand(d_out)
        ws = (w.float() * torch.cat((torch.ones_like(s), s))[:, None]).bfloat16()
        y, pre = lcn.lcn_gated_linear(x, ws, keep_pre=True)
        dx, dw, _ = lcn.lcn_gated_linear_backward(x, ws, pre, dy)
        want = oracle(x, ws, None, dy, "silu")
        for i in range(d_out):   # per column; its neighbours are up to 10^(12 * 8 / d_out) larger
            room = 2.0 ** -8 * 2 + 2.0 ** -14 * (4.0 if s.min() == s.max() else 10.0 ** (12 * 8 / (d_out - 1)))
            if room < 0.1:
                assert off(dw[i], want[3][i]) <= room and off(dw[d_out + i], want[3][d_out + i]) <= room


@pytest.mark.parametrize("rows", [3, 300])
def test_what_is_kept_may_be_infinite(rows):
    """A value that is not finite comes back as it is, and its neighbours with a rounding to 7 bits."""
    x, w, b, dy = inputs(rows, 40, 24, BF16)
    x[1, 3], x[2, 5] = math.inf, math.nan
    w[:, 3] = w[:, 3].abs()
    y, pre = lcn.lcn_gated_linear(x, w, bias=b, activation=lcn.ACT_NONE, keep_pre=True)
    dx, _, _ = lcn.lcn_gated_linear_backward(x, w, pre, dy, activation=lcn.ACT_NONE)
    assert torch.isinf(y[1]).all() and torch.isnan(y[2]).all() and torch.isfinite(y[0]).all() and torch.isfinite(dx[0]).all()
    assert not torch.isfinite(dx[1]).any() and torch.isnan(dx[2]).all()
    if rows > 3:
        assert torch.isfinite(dx[3:]).all()


def column_sizes(kind, d_out):
    """Factors of columns: one of eight far above its neighbours, or 2^-20 to 2^20 in any order."""
    s = torch.ones(d_out, device=DEV)
    if kind == "any":
        return (2.0 ** torch.linspace(-20, 20, d_out)[torch.randperm(d_out, generator=generator(d_out))]).to(DEV)
    s[3::8] = 2.0 ** kind
    return s


@pytest.mark.parametrize("kind", [0, 6, 10, 13, 16, 24, 40, -12, -30, -60, "any"])
@pytest.mark.parametrize("rows,d_out", [(3, 40), (3, 37), (20, 64), (300, 37), (300, 200), (700, 520)])
def test_what_is_kept_is_near_each_value(rows, d_out, kind):
    """u and g, which db is for a dy of 1 in one row and no activation: kept within 2^-10 of each value, whatever its neighbours are
    (2^-7 where they are more than 2^27 apart), formed in sums of 48 terms and rounded once in db."""
    x, w, b, dy = inputs(rows, 48, d_out, BF16)
    s = column_sizes(kind, d_out)
    w = (w.float() * torch.cat((s, s))[:, None]).bfloat16()
    _, pre = lcn.lcn_gated_linear(x, w, activation=lcn.ACT_NONE, keep_pre=True)
    z = x.double() @ w.double().t().contiguous()
    terms = x.double().abs() @ w.double().abs().t().contiguous()
    for r in {0, 1, rows // 2, rows - 1}:
        dy.zero_()
        dy[r] = 1.0
        db = lcn.lcn_gated_linear_backward(x, w, pre, dy, activation=lcn.ACT_NONE)[2].double()
        want = torch.cat((z[r, d_out:], z[r, :d_out]))
        near = 2.0 ** -24 * 48 * torch.cat((terms[r, d_out:], terms[r, :d_out]))
        # a piece's largest and least value, which decide how it is kept
        some = torch.nn.functional.pad(z[r].view(2, d_out), (0, -d_out % 8)).abs().view(2, -1, 8)
        apart = some.amax(2) / torch.where(some == 0.0, math.inf, some).amin(2) > 2.0 ** 27
        far = apart.flip(0)[:, :, None].expand(-1, -1, 8).reshape(2, -1)[:, :d_out].flatten()
        room = want.abs() * (2.0 ** -8 + torch.where(far, 2.0 ** -7, 2.0 ** -10)) * (1 + 2.0 ** -7) + 2 * near
        assert ((db - want).abs() <= room).all(), ((db - want).abs() / room).max()


@pytest.mark.parametrize("act,gates", [("none", True), ("silu", False)])
@pytest.mark.parametrize("rows,d_out", [(3, 40), (20, 64), (300, 37), (300, 200), (700, 520)])
@pytest.mark.parametrize("kind", [6, 10, 13, 16, "any"])
def test_gradients_beside_larger_columns(kind, rows, d_out, act, gates):
    """Rows of dW and db are as exact beside columns that are larger as elsewhere.  g and u are kept within `kept` of each value; dz is
    rounded once above 512 rows, dW and db are rounded once.  The rows of x are nearly at right angles (few rows) or their errors
    independent (many): 1.25 covers what adds up in dW.  In db the errors of its terms are independent, 0.43 of their bound
    in the root mean square, of u and through the slope: 3 covers five deviations."""
    x, w, _, dy = inputs(rows, 48, d_out, BF16)
    s = column_sizes(kind, d_out)
    w = (w.float() * torch.cat((s if gates else torch.ones_like(s), s))[:, None]).bfloat16()
    _, pre = lcn.lcn_gated_linear(x, w, activation=ACTS[act], keep_pre=True)
    _, dw, db = lcn.lcn_gated_linear_backward(x, w, pre, dy, activation=ACTS[act])
    want = oracle(x, w, None, dy, act)
    kept = 2.0 ** -7 if kind == "any" else 2.0 ** -10
    for i in range(2 * d_out):
        assert off(dw[i], want[3][i]) <= 2.5 * 2.0 ** -8 + 1.25 * kept, i
    g, u, d = want[1][:, :d_out].detach().requires_grad_(True), want[1][:, d_out:], dy.double()
    a = FUNCTIONS[act](g)
    (slope,) = torch.autograd.grad(a.sum(), g)
    dz = torch.cat((d * u * slope, d * a.detach()), 1)
    assert ((db.double() - want[4]).abs() <= 2.0 ** -8 * want[4].abs() + 3 * kept * dz.norm(dim=0)).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_out,shift", [(5, 136, 0), (300, 136, 0), (700, 136, 0), (300, 135, 0), (300, 136, 1)])
def test_single_gradients_and_same_bits(rows, d_out, shift, dtype):
    """dx, dw and db have the same bits whichever are asked for, and from call to call."""
    x, w, b, dy = inputs(rows, 72, d_out, dtype, shift)
    _, z = lcn.lcn_gated_linear(x, w, bias=b, keep_pre=True)
    want = lcn.lcn_gated_linear_backward(x, w, z, dy)
    for asked in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (0, 0, 0)):
        got = lcn.lcn_gated_linear_backward(x, w, z, dy, with_x=asked[0], with_w=asked[1], with_bias=asked[2])
        for a, u, v in zip(asked, got, want):
            assert torch.equal(u, v) if a else u is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [(5, 96, 136), (300, 33, 64), (300, 96, 136), (700, 96, 130)])
def test_operands_that_are_not_needed_may_be_missing(rows, d_in, d_out, dtype):
    """x is read for dW only, and W for dx only (the C entry point)."""
    from paper_2107_06876_amd import encoder
    x, w, b, dy = inputs(rows, d_in, d_out, dtype)
    _, z = lcn.lcn_gated_linear(x, w, bias=b, keep_pre=True)
    dx, dw, db = lcn.lcn_gated_linear_backward(x, w, z, dy)
    sizes = (rows, d_in, d_out, 0 if dtype == F32 else 1)
    space = torch.empty(encoder._bytes("lcn_gated_linear_workspace_bytes", (*sizes, 1)), dtype=torch.uint8, device=DEV)
    for with_x, with_w in ((True, False), (False, True), (False, False)):
        got = [torch.full_like(t, 7.0) for t in (dx, dw, db)]
        encoder._call("lcn_gated_linear_backward", x.device, x.data_ptr() if with_w else None, w.data_ptr() if with_x else None, z.data_ptr(),
                      dy.data_ptr(), *sizes, ACTS["silu"], got[0].data_ptr() if with_x else None, got[1].data_ptr() if with_w else None,
                      got[2].data_ptr(), space.data_ptr(), space.numel())
        narrow_by_planes = rows >= 128 and d_in <= 64 and d_out <= 64
        for u, v, asked in zip(got, (dx, dw, db), (with_x, with_w, True)):
            if not asked:
                assert (u == 7.0).all()
            elif narrow_by_planes:   # another way to the same sums
                assert off(u, v.double()) <= 2 * bound(dtype, max(rows, 2 * d_out), 1)
            else:
                assert torch.equal(u, v)


def test_differences():
    """<dy, y> changes along a direction as the gradients say (central differences of the float path)."""
    g = generator(14)
    x, w, b, dy = inputs(30, 20, 25, F32)
    for act in ("silu", "gelu", "tanh", "none"):
        _, pre = lcn.lcn_gated_linear(x, w, bias=b, activation=ACTS[act], keep_pre=True)
        grads = lcn.lcn_gated_linear_backward(x, w, pre, dy, activation=ACTS[act])
        for at, grad in enumerate(grads):
            step = normal(g, *grad.shape)
            h = 1e-3
            val = []
            for sign in (1, -1):
                args = [x, w, b]
                args[at] = args[at] + sign * h * step
                val.append((lcn.lcn_gated_linear(args[0], args[1], bias=args[2], activation=ACTS[act]).double() * dy.double()).sum())
            want = (grad.double() * step.double()).sum().item()
            # the third derivative times h^2, and the rounding of the values over h
            room = 2e-4 * grad.double().norm().item() * step.double().norm().item()
            assert abs((val[0] - val[1]).item() / (2 * h) - want) <= room


def test_no_rows():
    w, x = torch.ones(10, 4, device=DEV), torch.empty(0, 4, device=DEV)
    y, pre = lcn.lcn_gated_linear(x, w, keep_pre=True)
    assert y.shape == (0, 5) and pre.shape == (0,)
    dx, dw, db = lcn.lcn_gated_linear_backward(x, w, pre, y)
    assert dx.shape == (0, 4) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,d_in,d_out", [(6, 128, 256), (600, 128, 256), (900, 32, 64), (70, 2048, 40)])
def test_other_stream_and_graph(rows, d_in, d_out, dtype):
    x, w, b, dy = inputs(rows, d_in, d_out, dtype)

    def both():
        y, pre = lcn.lcn_gated_linear(x, w, bias=b, keep_pre=True)
        return (y, pre, *lcn.lcn_gated_linear_backward(x, w, pre, dy))

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
            t.fill_(77)
        both()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, want):
            assert torch.equal(u, v)


def test_refusals():
    x, w = torch.ones(4, 6, device=DEV), torch.ones(8, 6, device=DEV)
    for bad in (dict(x=x.t()), dict(x=x.half()), dict(x=x.bfloat16()), dict(w=torch.ones(8, 5, device=DEV)), dict(w=w[:7]),
                dict(x=x.cpu()), dict(bias=torch.ones(4, device=DEV)), dict(bias=torch.ones(8, device=DEV, dtype=BF16)),
                dict(out=torch.ones(4, 8, device=DEV)), dict(x=x[0])):
        with pytest.raises(ValueError):
            lcn.lcn_gated_linear(**dict(dict(x=x, w=w), **bad))
    with pytest.raises(lcn.LcnError):
        lcn.lcn_gated_linear(x, w, activation=9)
    with pytest.raises(lcn.LcnError):   # a workspace that is too small
        lcn.lcn_gated_linear(torch.ones(99, 6, device=DEV), w, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    _, pre = lcn.lcn_gated_linear(x, w, keep_pre=True)
    for bad in (dict(pre=pre[:-1]), dict(pre=pre.view(torch.float32)), dict(pre=pre.cpu()), dict(dy=torch.ones(4, 8, device=DEV))):
        with pytest.raises(ValueError):
            lcn.lcn_gated_linear_backward(**dict(dict(x=x, w=w, pre=pre, dy=torch.ones(4, 4, device=DEV)), **bad))
    with pytest.raises(lcn.LcnError):   # the gradient needs g and u
        lcn.lcn_gated_linear_backward(x, w, None, torch.ones(4, 4, device=DEV))

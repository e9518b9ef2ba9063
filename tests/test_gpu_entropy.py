"""lcn_cross_entropy and lcn_cross_entropy_backward against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, generator, normal, off

pytestmark = pytest.mark.gpu


def oracle(x, w, t, b, scale, grad):
    """loss, lse, dx, dw, db in 64 bits; rows with a negative target left out."""
    x, w = x.double(), w.double()
    z = scale * (x @ w.t().contiguous())
    if b is not None:
        z = z + b.double()
    lse = torch.logsumexp(z, 1)
    kept = t >= 0
    at = t.clamp(min=0)
    loss = torch.where(kept, lse - z.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    g = torch.where(kept, grad.double(), torch.zeros_like(lse))
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, at[:, None], -torch.ones_like(lse)[:, None])
    p = torch.where(kept[:, None], p * g[:, None], torch.zeros_like(p))
    xs = torch.where(kept[:, None], x, torch.zeros_like(x))
    return loss, lse, scale * (p @ w), scale * (p.t().contiguous() @ xs), p.sum(0)


def inputs(rows, vocab, dim, dtype, ignored=0.2, shift=0, bias=True):
    g = generator(rows, vocab, dim)
    x = normal(g, rows, dim, dtype=dtype, scale=dim ** -0.5, shift=shift)
    w = normal(g, vocab, dim, dtype=dtype, shift=shift)
    b = normal(g, vocab, scale=0.7) if bias else None
    t = torch.randint(0, vocab, (rows,), generator=g)
    t[torch.rand(rows, generator=g) < ignored] = -1
    if rows > 2:
        t[0], t[1] = vocab - 1, 0
    return x, w, t.to(DEV), b, torch.rand(rows, generator=g).to(DEV)


def check(rows, vocab, dim, dtype, scale=2.0, **how):
    print("entropy", rows, vocab, dim, dtype, how, flush=True)
    x, w, t, b, grad = inputs(rows, vocab, dim, dtype, **how)
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b, scale=scale)
    dx, dw, db = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b, scale=scale)
    eloss, else_, edx, edw, edb = oracle(x, w, t, b, scale, grad)
    # scores reach 10, a loss about log(vocab): an error of z counts up to ten times as much in p and in the loss
    assert off(lse, else_) <= 4 * bound(F32, dim)
    assert off(loss, eloss) <= 10 * bound(F32, dim)
    # the gradients' terms are off by p's own error as well
    more = 10 * bound(F32, dim)
    assert off(dx, edx) <= bound(dtype, vocab, 1) + more
    assert off(dw, edw) <= bound(dtype, rows, 1) + more
    assert (db is None) == (b is None)
    if b is not None:
        assert off(db, edb) <= bound(F32, rows) + more


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,dim", [
    (1, 1, 1), (1, 1000, 300), (2, 33, 64), (4, 5000, 16), (7, 777, 301), (8, 64, 8), (9, 64, 8), (9, 3, 5), (33, 1001, 300),
    (100, 257, 72), (300, 5003, 100), (1025, 777, 33), (64, 20000, 300)])
def test_sizes(rows, vocab, dim, dtype):
    check(rows, vocab, dim, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [3, 70])
def test_addresses_and_no_bias(rows, dtype):
    check(rows, 500, 64, dtype, shift=1)
    check(rows, 500, 64, dtype, bias=False, ignored=0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_tiles_and_pieces(dtype):
    """Enough rows and words that G takes several pieces of the vocabulary."""
    check(6000, 48000 if dtype == BF16 else 16001, 40, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [4, 80])
def test_rows_without_a_target_hold_anything(rows, dtype):
    """A row that is left out adds nothing to any gradient even where its x is infinite or not a number."""
    x, w, t, b, grad = inputs(rows, 300, 48, dtype)
    t[2] = -1
    t[3] = -100
    clean = x.clone()
    clean[2:4] = 0
    x[2] = math.nan
    x[3] = math.inf
    grad[3] = math.nan
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b)
    dx, dw, db = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b)
    assert loss[2] == 0 and loss[3] == 0 and not dx[2:4].any()
    _, l2 = lcn.lcn_cross_entropy(clean, w, t, bias=b)
    ex = lcn.lcn_cross_entropy_backward(clean, w, t, l2, grad, bias=b)
    for u, v in zip((dx, dw, db), ex):
        assert torch.isfinite(u).all() and torch.equal(u, v)


@pytest.mark.parametrize("rows", [5, 50])
def test_words_that_a_bias_takes_out(rows):
    x, w, t, b, grad = inputs(rows, 600, 32, F32, ignored=0.0)
    out = torch.zeros(600, dtype=torch.bool, device=DEV)
    out[:300] = True
    out[t] = False
    b = torch.where(out, torch.full_like(b, -math.inf), b)
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b)
    dx, dw, db = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b)
    e = oracle(x, w, t, b, 1.0, grad)
    for u, v in zip((loss, lse, dx, dw, db), e):
        assert off(u, v) <= 10 * bound(F32, 600)
    assert not dw[out].any() and not db[out].any()


@pytest.mark.parametrize("rows", [4, 40])
def test_targets_outside_the_vocabulary(rows):
    x, w, t, b, grad = inputs(rows, 100, 16, F32, ignored=0.0)
    t[1] = 100
    t[2] = 1 << 40
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b)
    bad = torch.zeros(rows, dtype=torch.bool, device=DEV)
    bad[1:3] = True
    assert torch.isnan(loss[bad]).all() and torch.isfinite(loss[~bad]).all() and torch.isfinite(lse).all()
    dx, _, _ = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all()


@pytest.mark.parametrize("rows", [3, 30])
def test_large_scores(rows):
    """Scores of several hundred: the maximum is taken out before any exponential."""
    x, w, t, b, grad = inputs(rows, 400, 24, F32, ignored=0.0)
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b, scale=400.0)
    e = oracle(x, w, t, b, 400.0, grad)
    assert off(lse, e[1]) <= 4 * bound(F32, 24) and off(loss, e[0]) <= 10 * bound(F32, 24)


def test_differences():
    """The loss along a direction changes as the gradients say (central differences of the float path)."""
    x, w, t, b, grad = inputs(40, 90, 20, F32)
    lse = lcn.lcn_cross_entropy(x, w, t, bias=b, scale=1.5)[1]
    grads = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b, scale=1.5)
    g = generator(5)
    for at, d in zip(range(3), grads):
        step = normal(g, *d.shape)
        h, val = 1e-3 if at else 4e-3, []
        for sign in (1, -1):
            args = [x, w, b]
            args[at] = args[at] + sign * h * step
            val.append((lcn.lcn_cross_entropy(args[0], args[1], t, bias=args[2], scale=1.5)[0].double() * grad.double()).sum())
        want = (d.double() * step.double()).sum().item()
        room = 2e-3 * d.double().norm().item() * step.double().norm().item()
        assert abs((val[0] - val[1]).item() / (2 * h) - want) <= room


def test_same_bits_other_stream_and_graph():
    x, w, t, b, grad = inputs(200, 3000, 64, BF16)

    def step():
        loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b)
        return (loss, lse, *lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b))

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    for u, v in zip(want, again):
        assert torch.equal(u, v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for u in got:
            u.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, v in zip(got, want):
            assert torch.equal(u, v)


def test_no_rows_and_single_gradients():
    x, w = torch.empty(0, 4, device=DEV), torch.ones(5, 4, device=DEV)
    t, none = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    loss, lse = lcn.lcn_cross_entropy(x, w, t)
    assert loss.shape == (0,) and lse.shape == (0,)
    dx, dw, db = lcn.lcn_cross_entropy_backward(x, w, t, lse, none, bias=torch.zeros(5, device=DEV))
    assert dx.shape == (0, 4) and not dw.any() and not db.any()
    x, w, t, b, grad = inputs(50, 200, 16, F32)
    lse = lcn.lcn_cross_entropy(x, w, t, bias=b)[1]
    both = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b)
    only_x = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b, with_w=False)
    only_w = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b, with_x=False)
    assert only_x[1] is None and only_w[0] is None
    assert torch.equal(only_x[0], both[0]) and torch.equal(only_w[1], both[1])


def test_refusals():
    x, w, t, b, grad = inputs(10, 20, 8, F32)
    for bad in (dict(x=x.t()), dict(w=w[:, :4]), dict(target=t.int()), dict(target=t[:5]), dict(bias=b.double()),
                dict(w=w.bfloat16()), dict(x=x.cpu())):
        args = dict(dict(x=x, w=w, target=t, bias=b), **bad)
        with pytest.raises(ValueError):
            lcn.lcn_cross_entropy(**args)
    for scale in (math.nan, math.inf):
        with pytest.raises(lcn.LcnError):
            lcn.lcn_cross_entropy(x, w, t, scale=scale)
    with pytest.raises(lcn.LcnError):
        lcn.lcn_cross_entropy(x, w, t, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))


def test_more_tiles_than_a_launch_has_in_one_dimension():
    """2^20 rows against more than 2^19 words: more than 2^32 threads in one launch of the scores' tiles."""
    g = generator(42)
    rows, vocab, dim = 1 << 20, (1 << 19) + 300, 8
    x, w = normal(g, rows, dim, dtype=BF16), normal(g, vocab, dim, dtype=BF16)
    t = torch.randint(0, vocab, (rows,), generator=g).to(DEV)
    loss, lse = lcn.lcn_cross_entropy(x, w, t)
    some = torch.tensor([0, 1, 255, 256, 70000, 524287, 524288, rows - 257, rows - 1], device=DEV)
    z = x[some].double() @ w.double().t().contiguous()
    want = torch.logsumexp(z, 1)
    assert torch.isfinite(loss).all()
    # 2049 tiles of 256 words: sums of 32-bit partial sums
    assert off(lse[some], want) <= bound(F32, vocab) and off(loss[some], want - z.gather(1, t[some, None])[:, 0]) <= bound(F32, vocab)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 3, 8, 30, 600])
@pytest.mark.parametrize("bias", [False, True])
def test_a_target_with_all_the_weight(rows, bias, dtype):
    """Scores of several hundred, the target's far above all others: the loss is 0 and not below, and no gradient is left."""
    g = generator(41, rows)
    vocab, dim, scale = 400, 24, 400.0
    w = normal(g, vocab, dim, dtype=dtype)
    t = torch.randint(0, vocab, (rows,), generator=g).to(DEV)
    x = w.double()[t]
    x = (x * (0.9 + 0.1 * torch.rand(rows, 1, generator=g).to(DEV)) / (x * x).sum(1, keepdim=True)).to(dtype)
    b = normal(g, vocab) if bias else None
    grad = (0.5 + torch.rand(rows, generator=g)).to(DEV)
    z = scale * (x.double() @ w.double().t().contiguous()) + (b.double() if bias else 0.0)
    at = z.gather(1, t[:, None])[:, 0]
    rest = z.scatter(1, t[:, None], -math.inf).max(1).values
    far = at - rest > 40.0   # the others' weight is below 400 e^-40
    t = torch.where(far, t, torch.full_like(t, -1))
    assert far.sum() >= 0.8 * rows
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b, scale=scale)
    assert (loss >= 0).all() and loss.max().item() <= 2.0 ** -24
    assert off(lse, torch.logsumexp(z, 1)) <= bound(F32, dim)
    dx, dw, db = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b, scale=scale)
    # one rounding of P = 1 in every row
    step = 2.0 ** -24 * 1.5 * scale
    assert dx.double().abs().max().item() <= step * w.double().abs().max().item()
    assert dw.double().abs().max().item() <= step * x.double().abs().max().item() * rows
    assert db is None or db.double().abs().max().item() <= 2.0 ** -24 * 1.5 * rows

"""lcn_attention and lcn_attention_backward against the formulas in 64 bits, set by set."""
import math

import pytest
import torch

import paper_2107_06876_amd as lcn
from operator_checks import BF16, DEV, F32, bound, generator, normal, off

pytestmark = pytest.mark.gpu


def offsets(lengths):
    return torch.tensor([0] + list(torch.tensor(lengths, dtype=torch.int64).cumsum(0)), dtype=torch.int64, device=DEV)


def oracle(q, k, v, do, nq, nk, scale, causal=False, prefix=None, slopes=None, cap=0.0):
    """o, lse, dq, dk, dv in 64 bits on the CPU; queries without a key give 0, -inf and no gradient."""
    q, k, v, do = (t.double().cpu() for t in (q, k, v, do))
    h, hk = q.shape[1], k.shape[1]
    o, lse = torch.zeros_like(q), torch.full((h, q.shape[0]), -math.inf, dtype=torch.float64)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    a = e = 0
    for p, (m, n) in enumerate(zip(nq, nk)):
        b, f = a + m, e + n
        pos, j = torch.arange(m)[:, None] + n - m, torch.arange(n)[None, :]
        seen = torch.ones(m, n, dtype=torch.bool)
        if causal:
            seen = (j <= pos) | (j < (int(prefix[p]) if prefix is not None else 0))
        for x in range(h if m and n else 0):
            y = x // (h // hk)
            Q, K, V, D = q[a:b, x], k[e:f, y], v[e:f, y], do[a:b, x]
            z = scale * Q @ K.t()
            cut = torch.ones_like(z)
            if cap > 0:
                t = torch.tanh(z / cap)
                z, cut = cap * t, 1 - t * t
            if slopes is not None:
                z = z - float(slopes[x]) * (pos - j).abs()
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            l = torch.logsumexp(z, 1)
            P = torch.where(seen, torch.exp(z - l[:, None]), torch.zeros_like(z))
            O = P @ V
            S = P * (D @ V.t() - (D * O).sum(1, keepdim=True)) * cut * scale
            o[a:b, x], lse[x, a:b], dq[a:b, x] = O, l, S @ K
            dk[e:f, y] += S.t() @ Q
            dv[e:f, y] += P.t() @ D
        a, e = b, f
    return tuple(t.to(DEV) for t in (o, lse, dq, dk, dv))


def check(nq, nk, heads, kv_heads, dim, dtype, causal=False, prefix=None, slopes=None, cap=0.0, shift=0, size=1.0, max_q=0):
    print("attention", list(nq)[:8], list(nk)[:8], heads, kv_heads, dim, dtype, causal, prefix, slopes, cap, shift, flush=True)
    g = generator(sum(nq), sum(nk), heads, dim)
    q = normal(g, sum(nq), heads, dim, dtype=dtype, shift=shift, scale=size)
    k = normal(g, sum(nk), kv_heads, dim, dtype=dtype, shift=shift, scale=size)
    v = normal(g, sum(nk), kv_heads, dim, dtype=dtype, shift=shift)
    do = normal(g, sum(nq), heads, dim, dtype=dtype, shift=shift)
    how = dict(causal=causal, cap=cap, prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=DEV),
               slopes=None if slopes is None else torch.tensor(slopes, device=DEV), max_q=max_q)
    qo, ko = offsets(nq), offsets(nk)
    o, lse = lcn.lcn_attention(q, k, v, qo, ko, **how)
    dq, dk, dv = lcn.lcn_attention_backward(q, k, v, o, lse, do, qo, ko, **how)
    want = oracle(q, k, v, do, nq, nk, dim ** -0.5, causal, prefix, slopes, cap)
    longest = max(max(nk, default=1), max(nq, default=1), 1)
    # scores up to about 10: their rounding counts ten times in P
    more = 10 * bound(F32, dim) if longest else 0.0
    assert off(o, want[0]) <= bound(dtype, longest, 1) + more
    assert off(lse, want[1]) <= bound(F32, dim + longest)
    # dS is a difference of numbers of the size of dP; o enters it as it was rounded
    terms = v.double().norm().item() * do.double().norm().item() * max(q.double().norm().item(), k.double().norm().item())
    for got, exact in zip((dq, dk, dv), want[2:]):
        room = bound(dtype, longest * heads // kv_heads, 2) + 4 * more
        if exact.norm().item() <= 1e-12 * terms:   # a single key: P = 1 and dP = delta, so dS is zero but for rounding
            assert got.double().norm().item() <= room * terms
        else:
            assert off(got, exact) <= room
    return o, lse, dq, dk, dv


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [1, 8, 20, 32, 64, 80, 100, 128])
def test_dims(dim, dtype):
    check([40, 17], [33, 70], 4, 2, dim, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq,nk", [
    ([1], [1]), ([0, 1, 0, 5], [3, 1, 0, 0]), ([64], [64]), ([65], [63]), ([128, 1], [129, 1]), ([200], [300]), ([300], [7]),
    ([3] * 70, [5] * 70), ([1, 500, 2], [257, 300, 1]), ([33] * 5 + [0] * 70 + [40], [33] * 5 + [0] * 70 + [40])])
def test_lengths(nq, nk, dtype):
    check(nq, nk, 2, 1, 32, dtype)
    check(nq, nk, 2, 2, 64, dtype, causal=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (6, 6), (8, 2), (5, 1)])
def test_heads(heads, kv_heads, dtype):
    check([70, 150], [70, 150], heads, kv_heads, 64, dtype, causal=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", [
    dict(causal=True, prefix=[20, 0, 500]), dict(causal=True, prefix=[64, 130, 1]), dict(slopes=[0.5, 0.01]),
    dict(causal=True, slopes=[0.3, 0.0]), dict(cap=5.0), dict(cap=2.0, causal=True, prefix=[7, 70, 0], slopes=[0.1, 0.2])])
def test_masks_and_scores(how, dtype):
    check([90, 140, 33], [90, 140, 33], 2, 1, 64, dtype, **how)
    check([10, 140, 64], [90, 150, 64], 2, 2, 32, dtype, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_queries_that_see_no_key(dtype):
    """Causal sets with more queries than keys: the first queries see nothing."""
    o, lse, dq, dk, dv = check([100, 5, 70], [30, 0, 69], 2, 1, 32, dtype, causal=True)
    assert not o[:70].any() and not dq[:70].any() and (lse[:, :70] == -math.inf).all() and not o[100:105].any()
    check([100, 5, 70], [30, 0, 69], 2, 1, 32, dtype, causal=True, prefix=[3, 2, 0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_addresses_of_one_element(dtype):
    check([50, 80], [60, 80], 2, 1, 64, dtype, shift=1)
    check([50, 80], [50, 80], 2, 2, 32, dtype, shift=3, causal=True, cap=4.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_sets(dtype):
    check([700, 1025], [1100, 1025], 4, 2, 128, dtype, causal=True)
    check([513], [2050], 2, 1, 64, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("max_q", [0, 1])
@pytest.mark.parametrize("how", [dict(), dict(causal=True), dict(causal=True, slopes=[0.02] * 8, cap=10.0)])
def test_single_queries(max_q, how, dtype):
    check([1] * 9, [1, 64, 65, 0, 3000, 17, 1111, 300, 5000], 8, 2, 64, dtype, max_q=max_q, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_few_queries(dtype):
    """Several queries per set over long keys, with the largest number given."""
    check([3, 0, 5, 1], [1000, 50, 4001, 5], 8, 2, 128, dtype, max_q=5, causal=True)
    check([20, 3], [2000, 700], 4, 4, 32, dtype, max_q=20)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_scores(dtype):
    """Scores in the hundreds: the running maximum keeps the exponentials in range."""
    g = generator(21)
    q, k, v = (normal(g, 150, 2, 32, dtype=dtype, scale=s) for s in (20.0, 20.0, 1.0))
    off_ = offsets([150])
    o, lse = lcn.lcn_attention(q, k, v, off_, off_)
    want = oracle(q, k, v, v, [150], [150], 32 ** -0.5)
    assert torch.isfinite(o).all() and off(lse, want[1]) <= bound(F32, 182)
    # scores of 500 are rounded by 2^-24 of that: an error of up to 2^-14 in P's exponent
    assert off(o, want[0]) <= bound(dtype, 150, 1) + 2.0 ** -12


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views_with_strides(dtype):
    """q, k and v as views of one projection, and of tensors with the heads first."""
    g = generator(22)
    lengths = [70, 33, 150]
    n = sum(lengths)
    qkv = normal(g, n, 3, 4, 32, dtype=dtype)
    off_ = offsets(lengths)
    do = normal(g, n, 4, 32, dtype=dtype)
    views = [qkv[:, i] for i in range(3)]
    whole = [t.contiguous() for t in views]
    first = [t.permute(1, 0, 2).contiguous().permute(1, 0, 2) for t in views]
    want = lcn.lcn_attention(*whole, off_, off_, causal=True)
    grads = lcn.lcn_attention_backward(*whole, *want, do, off_, off_, causal=True)
    for form in (views, first):
        got = lcn.lcn_attention(*form, off_, off_, causal=True)
        for u, w in zip((*got, *lcn.lcn_attention_backward(*form, *got, do, off_, off_, causal=True)), (*want, *grads)):
            assert torch.equal(u, w)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq", [[3, 0, 90], [1, 1, 1]])
def test_other_tokens_hold_anything(nq, dtype):
    """Tokens outside every set, and keys of other sets, may be infinite or not numbers."""
    g = generator(23, sum(nq))
    nk = [70, 40, 100]
    q, k, v = normal(g, sum(nq), 2, 64, dtype=dtype), normal(g, 250, 2, 64, dtype=dtype), normal(g, 250, 2, 64, dtype=dtype)
    do = normal(g, sum(nq), 2, 64, dtype=dtype)
    qo, ko = offsets(nq), offsets(nk)
    most = max(nq) if max(nq) < 4 else 0
    want = lcn.lcn_attention(q, k, v, qo, ko, max_q=most)
    grads = lcn.lcn_attention_backward(q, k, v, *want, do, qo, ko)
    k2, v2 = k.clone(), v.clone()
    k2[210:], v2[210:] = math.nan, math.inf
    if nq[1] == 0:
        k2[70:110], v2[70:110] = math.inf, math.nan
    got = lcn.lcn_attention(q, k2, v2, qo, ko, max_q=most)
    for u, w in zip(got, want):
        assert torch.equal(u, w)
    dq, dk, dv = lcn.lcn_attention_backward(q, k2, v2, *got, do, qo, ko)
    assert torch.equal(dq, grads[0])
    for s in (slice(0, 70), slice(110, 210)):
        assert torch.equal(dk[s], grads[1][s]) and torch.equal(dv[s], grads[2][s])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", [dict(), dict(causal=True, prefix=[900, 0]), dict(cap=5.0), dict(slopes=[0.01, 0.2], cap=60.0)])
def test_few_tiles_over_long_sets(how, dtype):
    """Few tiles: the keys of a query tile and the queries of a key tile are split over workgroups."""
    check([150, 20], [3000, 1111], 2, 1, 32, dtype, **how)
    check([2100, 700], [60, 500], 2, 2, 64, dtype, **how)


def test_a_prefix_without_a_causal_mask_changes_nothing():
    g = generator(30)
    q, off_ = normal(g, 90, 2, 32), offsets([40, 50])
    a = lcn.lcn_attention(q, q, q, off_, off_)
    b = lcn.lcn_attention(q, q, q, off_, off_, prefix=torch.tensor([5, 7], dtype=torch.int32, device=DEV))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_differences():
    """<do, o> along a direction changes as the gradients say (central differences of the float path)."""
    g = generator(24)
    nq, nk = [20, 45], [30, 45]
    q, k, v = normal(g, 65, 4, 16), normal(g, 75, 2, 16), normal(g, 75, 2, 16)
    do = normal(g, 65, 4, 16)
    qo, ko = offsets(nq), offsets(nk)
    how = dict(causal=True, cap=3.0, slopes=torch.tensor([0.1, 0.2, 0.0, 0.3], device=DEV))
    o, lse = lcn.lcn_attention(q, k, v, qo, ko, **how)
    grads = lcn.lcn_attention_backward(q, k, v, o, lse, do, qo, ko, **how)
    for at, grad in zip(range(3), grads):
        step = normal(g, *grad.shape)
        h, val = 1e-3, []
        for sign in (1, -1):
            args = [q, k, v]
            args[at] = args[at] + sign * h * step
            val.append((lcn.lcn_attention(*args, qo, ko, **how)[0].double() * do.double()).sum())
        want = (grad.double() * step.double()).sum().item()
        room = 2e-3 * grad.double().norm().item() * step.double().norm().item()
        assert abs((val[0] - val[1]).item() / (2 * h) - want) <= room


def test_offsets_beyond_the_tensors_are_cut():
    g = generator(25)
    q, k, v = normal(g, 50, 1, 32), normal(g, 60, 1, 32), normal(g, 60, 1, 32)
    o, _ = lcn.lcn_attention(q, k, v, torch.tensor([0, 20, 900], device=DEV), torch.tensor([0, 30, 1 << 40], device=DEV))
    w, _ = lcn.lcn_attention(q, k, v, offsets([20, 30]), offsets([30, 30]))
    assert torch.equal(o, w)


def test_same_bits_other_stream_and_graph():
    g = generator(26)
    lengths = [100, 1, 260]
    q, k, v = (normal(g, 361, h, 64, dtype=BF16) for h in (4, 2, 2))
    do, off_ = normal(g, 361, 4, 64, dtype=BF16), offsets(lengths)
    single, one = normal(g, 3, 4, 64, dtype=BF16), offsets([1, 1, 1])

    def step():
        o, lse = lcn.lcn_attention(q, k, v, off_, off_, causal=True)
        return (o, lse, *lcn.lcn_attention_backward(q, k, v, o, lse, do, off_, off_, causal=True),
                *lcn.lcn_attention(single, k, v, one, off_, max_q=1))

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = step()
    side.synchronize()
    for u, w in zip(want, again):
        assert torch.equal(u, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for u in got:
            u.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for u, w in zip(got, want):
            assert torch.equal(u, w)


def test_nothing_to_do():
    e = torch.empty(0, 2, 32, device=DEV)
    z = torch.zeros(3, dtype=torch.int64, device=DEV)
    o, lse = lcn.lcn_attention(e, e, e, z, z)
    assert o.shape == (0, 2, 32) and lse.shape == (2, 0)
    k = torch.ones(4, 2, 32, device=DEV)
    _, dk, dv = lcn.lcn_attention_backward(e, k, k, o, lse, e, z, offsets([4, 0]))
    assert not dk.any() and not dv.any()


def test_refusals():
    q, o = torch.ones(6, 4, 32, device=DEV), offsets([6])
    k = torch.ones(6, 2, 32, device=DEV)
    for bad in (dict(q=q.half()), dict(k=k.bfloat16()), dict(v=k[:5]), dict(q=q.transpose(1, 2)), dict(q=q[:, :3]), dict(q=q.cpu()),
                dict(q_off=o.int()), dict(k_off=offsets([3, 3])), dict(slopes=torch.ones(3, device=DEV)), dict(q=q[0]),
                dict(prefix=torch.ones(2, dtype=torch.int32, device=DEV)), dict(k=k[:1].expand(6, 2, 32))):
        args = dict(dict(q=q, k=k, v=k, q_off=o, k_off=o), **bad)
        with pytest.raises(ValueError):
            lcn.lcn_attention(**args)
    wide = torch.ones(6, 2, 160, device=DEV)
    for args, how in (((wide, wide, wide), {}), ((q, k, k), dict(scale=math.nan)), ((q, k, k), dict(cap=-1.0)),
                      ((q, k, k), dict(max_q=-1))):
        with pytest.raises(lcn.LcnError):
            lcn.lcn_attention(*args, o, o, **how)
    out, lse = lcn.lcn_attention(q, k, k, o, o)
    with pytest.raises(lcn.LcnError):
        lcn.lcn_attention_backward(q, k, k, out, lse, q, o, o, workspace=torch.empty(4, dtype=torch.uint8, device=DEV))


def test_more_workgroups_than_a_launch_has_in_one_dimension():
    """2^24 sets, nearly all empty: more than 2^32 threads."""
    sets = 1 << 24
    g = generator(35)
    q, k, v, do = (normal(g, 300, 1, 32, dtype=BF16) for _ in range(4))
    long_off = torch.zeros(sets + 1, dtype=torch.int64, device=DEV)
    long_off[sets // 2 + 1:] = 100
    long_off[sets:] = 300
    short = offsets([100, 200])
    want = lcn.lcn_attention(q, k, v, short, short)
    got = lcn.lcn_attention(q, k, v, long_off, long_off)
    for u, w in zip((*got, *lcn.lcn_attention_backward(q, k, v, *got, do, long_off, long_off)),
                    (*want, *lcn.lcn_attention_backward(q, k, v, *want, do, short, short))):
        assert torch.equal(u, w)


def test_more_rows_to_join_than_a_launch_has_in_one_dimension():
    """One query of 32 heads in each of more than 2^21 sets: the chunks of more than 2^26 rows are joined by a wavefront each."""
    sets, heads, nk, dim = (1 << 21) + 77, 32, 128, 8
    g = torch.Generator(device=DEV)
    g.manual_seed(36)
    q, k = (torch.randn(n, h, dim, generator=g, device=DEV, dtype=BF16) for n, h in ((sets, heads), (sets * nk, 1)))
    steps = torch.arange(sets + 1, device=DEV)
    o, lse = lcn.lcn_attention(q, k, k, steps, steps * nk, max_q=1)
    for p in (0, 1, sets // 3, (1 << 21) - 1, 1 << 21, sets - 1):
        part = slice(p * nk, (p + 1) * nk)
        want = oracle(q[p:p + 1], k[part], k[part], q[p:p + 1], [1], [nk], dim ** -0.5)
        assert off(o[p:p + 1], want[0]) <= bound(BF16, nk, 1) and off(lse[:, p:p + 1], want[1]) <= bound(F32, nk)


# ---- exactness ------------------------------------------------------------------


def one_head(q, k, scale):
    """lse in 64 bits of one head's queries against all keys, on the device."""
    z = scale * (q.double() @ k.double().t().contiguous())
    return torch.logsumexp(z, 1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_long_row_of_scores_is_not_scaled_by_rounding(dim, dtype):
    """8192 keys, scores of deviation 10: other queries' new maxima leave a query's sum alone.  q and k hold small whole numbers, so that
    q . k is exact; what is left is a rounding of lse itself (2^-25 of the power of two above it) and the sum's, which are smaller
    taken together than 2^-24 of the largest lse."""
    g = generator(31, dim)
    heads, nq, nk = 64, 1024, 8192   # so many tiles that no query's keys are split over workgroups
    q = normal(g, nq, heads, dim, scale=10.0).round().to(dtype)
    k = normal(g, nk, 1, dim).round().to(dtype)
    _, lse = lcn.lcn_attention(q, k, k, offsets([nq]), offsets([nk]))
    err, most = 0.0, 0.0
    for h in (0, 17, 40, 63):
        want = one_head(q[:, h], k[:, 0], dim ** -0.5)
        err += (lse[h].double() - want).square().sum().item()
        most = max(most, want.abs().max().item())
    assert math.sqrt(err / (4 * nq)) <= 2.0 ** -24 * most


@pytest.mark.parametrize("end", [1.0, -1.0])
@pytest.mark.parametrize("cap", [30.0, 40.0])
@pytest.mark.parametrize("how", [dict(), dict(causal=True, prefix=[40, 300])])
def test_scores_at_either_end_of_the_cap(end, cap, how):
    """All scores at +cap or at -cap and small v: the exponentials are not so small that v loses bits."""
    g = generator(32)
    lengths, dim = [100, 333], 64
    n = sum(lengths)
    q = (normal(g, n, 2, dim).abs() + 8.0).to(BF16)
    k = (end * (normal(g, n, 1, dim).abs() + 8.0)).to(BF16)
    v, do = normal(g, n, 1, dim, dtype=BF16, scale=2.0 ** -32), normal(g, n, 2, dim, dtype=BF16)
    prefix = how.get("prefix")
    args = dict(how, cap=cap, prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=DEV))
    o, lse = lcn.lcn_attention(q, k, v, offsets(lengths), offsets(lengths), **args)
    want = oracle(q, k, v, do, lengths, lengths, dim ** -0.5, how.get("causal", False), prefix, None, cap)
    assert off(o, want[0]) <= bound(BF16, 333, 1) + 2.0 ** -21 * cap
    assert off(lse, want[1]) <= bound(F32, 333)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", [dict(), dict(causal=True, cap=5.0), dict(slopes=[0.1, 0.2])])
def test_gradients_of_keys_without_those_of_queries(how, dtype):
    """dk and dv, and dq, have the same bits whichever are asked for."""
    g = generator(33)
    nq, nk = [90, 140, 33, 700], [90, 140, 33, 900]
    for dim, shift in ((64, 0), (20, 0), (64, 1)):
        q, do = (normal(g, sum(nq), 2, dim, dtype=dtype, shift=shift) for _ in range(2))
        k, v = (normal(g, sum(nk), 1, dim, dtype=dtype, shift=shift) for _ in range(2))
        args = dict(how, slopes=None if "slopes" not in how else torch.tensor(how["slopes"], device=DEV))
        qo, ko = offsets(nq), offsets(nk)
        kept = lcn.lcn_attention(q, k, v, qo, ko, **args)
        all_three = lcn.lcn_attention_backward(q, k, v, *kept, do, qo, ko, **args)
        dq, none_k, none_v = lcn.lcn_attention_backward(q, k, v, *kept, do, qo, ko, with_kv=False, **args)
        none_q, dk, dv = lcn.lcn_attention_backward(q, k, v, *kept, do, qo, ko, with_q=False, **args)
        assert none_q is None and none_k is None and none_v is None
        for u, w in zip((dq, dk, dv), all_three):
            assert torch.equal(u, w)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("max_q", [0, 2])
@pytest.mark.parametrize("nq,nk", [([1, 2, 1], [300, 900, 5]), ([70, 200], [70, 200])])
def test_tokens_in_no_set(nq, nk, max_q, dtype):
    """Before the first and behind the last set: o and all gradients are zero, lse is -inf."""
    if max(nq) > 2:
        max_q = 0
    g = generator(34)
    before, behind = 37, 150
    q, do = (normal(g, before + sum(nq) + behind, 4, 64, dtype=dtype) for _ in range(2))
    k, v = (normal(g, before + sum(nk) + behind, 2, 64, dtype=dtype) for _ in range(2))
    qo, ko = offsets(nq) + before, offsets(nk) + before
    for t in (q, k):   # what torch hands out next has been used
        for _ in range(4):
            torch.full(t.shape, 7.0, dtype=dtype, device=DEV)
    torch.full((4, q.shape[0]), 7.0, device=DEV)
    o, lse = lcn.lcn_attention(q, k, v, qo, ko, max_q=max_q)
    dq, dk, dv = lcn.lcn_attention_backward(q, k, v, o, lse, do, qo, ko, max_q=max_q)
    for t, n in ((o, sum(nq)), (dq, sum(nq)), (dk, sum(nk)), (dv, sum(nk))):
        assert not t[:before].any() and not t[before + n:].any() and t[before:before + n].any()
    assert (lse[:, :before] == -math.inf).all() and (lse[:, before + sum(nq):] == -math.inf).all()
    none = torch.zeros(1, dtype=torch.int64, device=DEV)   # no sets at all
    o, lse = lcn.lcn_attention(q, k, v, none, none, max_q=max_q)
    grads = lcn.lcn_attention_backward(q, k, v, o, lse, do, none, none, max_q=max_q)
    assert not o.any() and (lse == -math.inf).all() and not any(t.any() for t in grads)


def test_tokens_in_no_set_of_a_caller_that_keeps_them():
    """Without `clear` the C entry points leave such tokens' memory alone: two calls may share an output."""
    import ctypes
    from paper_2107_06876_amd import encoder
    g = generator(38)
    q, do = (normal(g, 200, 2, 64) for _ in range(2))
    o, dq, dk, dv = (torch.full_like(q, 7.0) for _ in range(4))
    lse = torch.full((2, 200), 7.0, device=DEV)
    off_ = torch.tensor([30, 100, 150], device=DEV)
    for clear in (0, 1):
        d = encoder._attention_desc(q, q, q, off_, off_, None, False, None, None, 0.0, 0)
        d.clear = clear
        for back in (0, 1):
            at, size, space = encoder._attention_space(d, back, None, q.device)
            more = ((o, lse, do, dq, dk, dv) if back else (o, lse))
            encoder._call("lcn_attention_backward" if back else "lcn_attention", q.device, ctypes.byref(d), q.data_ptr(), q.data_ptr(),
                          q.data_ptr(), *(t.data_ptr() for t in more), at, size)
        for t in (o, dq, dk, dv):
            assert (t[:30] == 7.0 * (1 - clear)).all() and (t[150:] == 7.0 * (1 - clear)).all() and (t[30:150] != 7.0).any()
        left = -math.inf if clear else 7.0
        assert (lse[:, :30] == left).all() and (lse[:, 150:] == left).all() and torch.isfinite(lse[:, 30:150]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_more_queries_than_max_q_says(dtype):
    """What a hint below the truth leaves out is not a number, and not what the memory held."""
    g = generator(39)
    q, k = normal(g, 8, 4, 64, dtype=dtype), normal(g, 2000, 2, 64, dtype=dtype)
    qo, ko = offsets([2, 5, 1]), offsets([700, 800, 500])
    for _ in range(4):
        torch.full(q.shape, 7.0, dtype=dtype, device=DEV)
        torch.full((4, 8), 7.0, device=DEV)
    o, lse = lcn.lcn_attention(q, k, k, qo, ko, max_q=2)
    want, l = lcn.lcn_attention(q, k, k, qo, ko, max_q=5)
    kept = torch.tensor([0, 1, 2, 3, 7], device=DEV)
    assert torch.equal(o[kept], want[kept]) and torch.equal(lse[:, kept], l[:, kept])
    assert torch.isnan(o[4:7]).all() and torch.isnan(lse[:, 4:7]).all()


# ---- forms that the tests above leave out ------------------------------------------


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,shift", [(1, 0), (20, 0), (100, 0), (64, 1), (128, 1)])
@pytest.mark.parametrize("how", [dict(), dict(causal=True, prefix=[4, 2500, 0, 500])])
def test_new_tokens_without_whole_pieces(how, dim, shift, dtype):
    """Keys split over workgroups, read one value at a time: odd widths and addresses, also behind a prefix."""
    check([1, 3, 2, 3], [129, 3000, 64, 700], 8, 2, dim, dtype, shift=shift, max_q=3, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", [dict(causal=True, prefix=[900, 0, 1]), dict(causal=True, prefix=[1000, 3, 650], cap=20.0, slopes=[0.01] * 8)])
def test_new_tokens_behind_a_prefix(how, dtype):
    check([4, 2, 1], [1000, 400, 700], 8, 2, 64, dtype, max_q=4, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,shift", [(33, 0), (7, 0), (64, 1), (65, 3)])
@pytest.mark.parametrize("how", [dict(), dict(causal=True)])
def test_few_tiles_without_whole_pieces(how, dim, shift, dtype):
    """Sums of several workgroups whose rows are no whole pieces, and whose number is odd."""
    check([151], [3001], 1, 1, dim, dtype, shift=shift, **how)
    check([2501], [151], 3, 1, dim, dtype, shift=shift, **how)


@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("cap", [3.0, 30.0, 39.5, 50.0])
@pytest.mark.parametrize("how", [dict(), dict(causal=True), dict(causal=True, prefix=[20, 400, 0])])
def test_capped_documents(how, cap, dim):
    """Caps on whole rows of bf16, under all masks and at all widths."""
    check([90, 500, 33], [90, 500, 33], 4, 1, dim, BF16, cap=cap, size=2.0, **how)
    check([90, 140, 33], [300, 700, 33], 2, 2, dim, BF16, cap=cap, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_peaked_softmax_over_many_keys(dtype):
    """Steep slopes: the weight of a row lies on few of its 1000 keys, and o is as large as one v."""
    check([1000], [1000], 2, 1, 64, dtype, causal=True, slopes=[4.0, 1.0])

"""How often results of bf16 tensors are rounded on their way: in the 2-norm, where one rounding too many shows, and value by value."""
import pytest
import torch

import paper_2107_06876_amd as lcn
import test_gpu_attention as attention
import test_gpu_entropy as entropy
import test_gpu_linear as linear
from operator_checks import BF16, DEV, farthest, generator, normal, off, roundings

pytestmark = pytest.mark.gpu


def near(got, want, rounded, what):
    """`rounded` roundings in the 2-norm, and no value far off."""
    o, f = off(got, want), farthest(got, want)
    print(what, o / roundings(1) * 1.1, f, flush=True)
    assert o <= roundings(rounded) and f <= 1.0


@pytest.mark.parametrize("rows", [12, 300, 512, 700, 4103])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_linear(act, rows):
    """Up to 512 rows dz keeps a second plane, so that dx and dw are rounded once; above, dz is rounded as well."""
    d_in, d_out = (264, 520) if rows < 4000 else (512, 4096)
    g = generator(51, rows)
    x, w = normal(g, rows, d_in, dtype=BF16), normal(g, d_out, d_in, dtype=BF16, scale=d_in ** -0.5)
    b, r, dy = normal(g, d_out, dtype=BF16), normal(g, rows, d_out, dtype=BF16), normal(g, rows, d_out, dtype=BF16)
    y, z = lcn.lcn_linear(x, w, bias=b, residual=r, activation=linear.ACTS[act], keep_pre=True)
    grads = lcn.lcn_linear_backward(x, w, z, dy, activation=linear.ACTS[act])
    want = linear.oracle(x, w, b, r, dy, act)
    near(y, want[0], 1, "y")
    once = 1 if rows <= 512 or act == "none" else 2
    for got, exact, n, what in zip(grads, want[2:], (once, once, 1), ("dx", "dw", "db")):
        near(got, exact, n, what)


@pytest.mark.parametrize("rows", [5, 40, 512, 600, 3000])
def test_cross_entropy(rows):
    """Up to 512 rows G keeps a second plane; above, it is rounded, but in dx not the part that is most of it, the target's."""
    vocab, dim = 700, 136
    x, w, t, b, grad = entropy.inputs(rows, vocab, dim, BF16)
    loss, lse = lcn.lcn_cross_entropy(x, w, t, bias=b, scale=2.0)
    dx, dw, db = lcn.lcn_cross_entropy_backward(x, w, t, lse, grad, bias=b, scale=2.0)
    want = entropy.oracle(x, w, t, b, 2.0, grad)
    near(dx, want[2], 1, "dx")
    near(dw, want[3], 1 if rows <= 512 else 2, "dw")


@pytest.mark.parametrize("dim", [32, 64, 128])
@pytest.mark.parametrize("how", [dict(), dict(causal=True), dict(cap=20.0), dict(slopes=[0.05, 0.1])])
def test_attention_over_short_sets(how, dim):
    """v far from its differences: o is large beside dS, whose sum with it is formed before o is rounded.  P is rounded in o and dv,
    dS in dq and dk."""
    g = generator(52, dim)
    lengths = [250, 33, 128, 200]
    n = sum(lengths)
    q, k, do = normal(g, n, 2, dim, dtype=BF16), normal(g, n, 1, dim, dtype=BF16), normal(g, n, 2, dim, dtype=BF16)
    v = (8.0 + normal(g, n, 1, dim)).to(BF16)
    off_ = attention.offsets(lengths)
    args = dict(how, slopes=None if "slopes" not in how else torch.tensor(how["slopes"], device=DEV))
    o, lse = lcn.lcn_attention(q, k, v, off_, off_, **args)
    got = lcn.lcn_attention_backward(q, k, v, o, lse, do, off_, off_, **args)
    want = attention.oracle(q, k, v, do, lengths, lengths, dim ** -0.5, how.get("causal", False), None, how.get("slopes"),
                            how.get("cap", 0.0))
    near(o, want[0], 2, "o")
    for u, e, what in zip(got, want[2:], ("dq", "dk", "dv")):
        # a query with a single key has no gradient but for rounding of its terms
        some = slice(None) if what == "dv" or not how.get("causal") else torch.tensor(
            [i for a, m in zip([0, 250, 283, 411], lengths) for i in range(a + (8 if what == "dq" else 0), a + m - 8)], device=DEV)
        near(u[some], e[some], 2, what)


@pytest.mark.parametrize("how", [dict(), dict(causal=True)])
def test_attention_over_long_sets(how):
    """Beyond 256 keys o enters dS as it was rounded."""
    g = generator(53)
    nq, nk = [500, 700], [1100, 700]
    q, do = (normal(g, 1200, 4, 64, dtype=BF16) for _ in range(2))
    k, v = (normal(g, 1800, 2, 64, dtype=BF16) for _ in range(2))
    qo, ko = attention.offsets(nq), attention.offsets(nk)
    o, lse = lcn.lcn_attention(q, k, v, qo, ko, **how)
    got = lcn.lcn_attention_backward(q, k, v, o, lse, do, qo, ko, **how)
    want = attention.oracle(q, k, v, do, nq, nk, 64 ** -0.5, how.get("causal", False))
    late = slice(0, 500)   # queries of the first set see 600 keys at least
    near(o[late], want[0][late], 2, "o")
    near(got[0][late], want[2][late], 3, "dq")
    near(got[2], want[4], 2, "dv")
    near(got[1][1100:], want[3][1100:], 3, "dk")

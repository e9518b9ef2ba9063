"""The work that is timed of the operators that produce and train embeddings: a matrix product with bias,
activation and residual; attention inside ragged sets; softmax cross entropy over a large vocabulary.

A case is a dict of plain values; `listed()` has the fixed ones, `draw(rng)` makes more of the same ranges,
`prepare` makes what a program holds before the call, `run` is one pass, `work` what a pass cannot do
without, `exact` the result in 64 bits.  With `own` false a pass uses elementary torch operations in 32 bits,
with `own` true the library's entry points.

  linear         y = act(x W^T + b) + r; a training pass also returns the gradients of x, W and b for a given dy
  attention      softmax over the keys of a query's own set, by offsets; scores may be capped by a tanh, get a
                 bias -slope |distance| per head, be causal with a prefix that every query sees; a training pass
                 also returns the gradients of q, k and v
  cross_entropy  loss = logsumexp(scale x W^T + b) - (the target's score), rows with a negative target left out;
                 a training pass also returns the gradients of x, W and b
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _linear(name, rows, d_in, d_out, act, dtype, train, residual=False, bias=True):
    c = dict(kind="linear", rows=rows, d_in=d_in, d_out=d_out, act=act, dtype=dtype, train=train, residual=residual,
             bias=bias)
    return dict(c, name=name) if name else c


def _attention(name, sets, q_lo, q_hi, k_lo, k_hi, heads, kv_heads, dim, dtype, train, causal=False, prefix=0,
               slopes=False, cap=0.0, cross=False):
    c = dict(kind="attention", sets=sets, q_lo=q_lo, q_hi=q_hi, k_lo=k_lo, k_hi=k_hi, heads=heads, kv_heads=kv_heads,
             dim=dim, dtype=dtype, train=train, causal=causal, prefix=prefix, slopes=slopes, cap=cap, cross=cross)
    return dict(c, name=name) if name else c


def _entropy(name, rows, vocab, dim, dtype, train, bias=False, ignored=0.0):
    c = dict(kind="cross_entropy", rows=rows, vocab=vocab, dim=dim, dtype=dtype, train=train, bias=bias,
             ignored=ignored)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token through a wide layer: every weight is read once
        _linear("token_bf16", 1, 2048, 8192, "silu", "bf16", False),
        # the tanh layer in front of a batch of 1024 graph pairs, some 40 nodes each, 32 wide (configuration 4)
        _linear("graph_nodes_f32", 40961, 32, 32, "tanh", "f32", False),
        # a training step of a layer on word embeddings (20 000 of width 300, configuration 3)
        _linear("words_train_f32", 20000, 300, 512, "tanh", "f32", True),
        # a training step of a wide layer with its residual; an odd number of rows
        _linear("wide_train_bf16", 16391, 1024, 4096, "gelu", "bf16", True, residual=True),
        # scoring one word against a vocabulary of 20 000 (configuration 3)
        _entropy("score_word_f32", 1, 20000, 300, "f32", False),
        # a training step of a supervised alignment: 5000 dictionary pairs against 20 000 words
        _entropy("dictionary_train_f32", 5000, 20000, 300, "f32", True, bias=True),
        # a training step of wide embeddings against a ragged vocabulary; a tenth of the rows has no target
        _entropy("wide_vocabulary_train_bf16", 4099, 50021, 1024, "bf16", True, ignored=0.1),
        # the vocabulary of configuration 5, bfloat16
        _entropy("large_vocabulary_train_bf16", 8192, 200000, 300, "bf16", True),
        # nodes of 1024 small graphs that attend to their own graph, near ones more (configuration 4), training
        _attention("graphs_train_f32", 1024, 16, 64, 16, 64, 4, 4, 32, "f32", True, slopes=True),
        # documents packed into one batch: causal behind a prefix, scores capped, shared key heads, training
        _attention("documents_train_bf16", 6, 500, 5000, 500, 5000, 16, 4, 128, "bf16", True, causal=True, prefix=100,
                   cap=30.0),
        # one new token for each of 32 sequences with contexts of all lengths
        _attention("new_tokens_bf16", 32, 1, 1, 100, 16000, 32, 8, 128, "bf16", False, causal=True),
        # two long sets that attend to a long partner each, forward
        _attention("long_pairs_bf16", 2, 8191, 8192, 8000, 8191, 16, 16, 64, "bf16", False, cross=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    limit = max(work(c)["flops"] for c in listed())
    room = max(_scores(c) for c in listed())
    while True:
        c = rng.choice([_draw_linear, _draw_attention, _draw_entropy])(rng)
        if work(c)["flops"] <= limit and _scores(c) <= room:
            return c


def _scores(c):
    """Numbers that a plain pass keeps at once."""
    if c["kind"] == "attention":
        q, k = _lengths(c)
        return c["sets"] * c["heads"] * max(q) * max(k)
    if c["kind"] == "linear":
        return c["rows"] * c["d_out"]
    return c["rows"] * c["vocab"]


def _draw_linear(rng):
    small = rng.random() < 0.4
    return _linear(None, _log_int(rng, 1, 64) if small else _log_int(rng, 64, 40000),
                   rng.choice([_log_int(rng, 16, 2048), 8 * _log_int(rng, 4, 256), 300]),
                   rng.choice([_log_int(rng, 16, 3000), 8 * _log_int(rng, 4, 300), 4096]),
                   rng.choice(["none", "tanh", "relu", "gelu", "silu"]), rng.choice(["f32", "bf16"]),
                   rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.8)


def _draw_attention(rng):
    what = rng.choice(["graphs", "documents", "tokens", "pairs"])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    dtype = rng.choice(["f32", "bf16"])
    if what == "graphs":
        lo = rng.randint(1, 24)
        return _attention(None, _log_int(rng, 16, 2048), lo, rng.randint(40, 64), lo, 64, heads, kv,
                          rng.choice([8, 16, 20, 32, 64]), dtype, rng.random() < 0.6, slopes=rng.random() < 0.5)
    if what == "documents":
        lo = _log_int(rng, 16, 1000)
        hi = lo + _log_int(rng, 16, 3000)
        return _attention(None, rng.randint(1, 8), lo, hi, lo, hi, heads, kv, rng.choice([32, 64, 80, 128]), dtype,
                          rng.random() < 0.6, causal=rng.random() < 0.7, prefix=rng.choice([0, 0, lo // 2]),
                          slopes=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 20.0, 50.0]))
    if what == "tokens":
        hi = _log_int(rng, 200, 16000)
        return _attention(None, _log_int(rng, 1, 64), 1, 1, rng.randint(1, hi // 2), hi, heads, kv,
                          rng.choice([32, 64, 128]), dtype, False, causal=True, slopes=rng.random() < 0.3,
                          cap=rng.choice([0.0, 30.0]))
    q, k = _log_int(rng, 100, 8000), _log_int(rng, 100, 8000)
    return _attention(None, rng.randint(1, 4), q, q + q // 8, k, k + k // 8, heads, kv, rng.choice([32, 64, 100, 128]),
                      dtype, rng.random() < 0.5, cross=True, cap=rng.choice([0.0, 30.0]))


def _draw_entropy(rng):
    small = rng.random() < 0.3
    rows = _log_int(rng, 1, 64) if small else _log_int(rng, 64, 10000)
    return _entropy(None, rows, _log_int(rng, 1000, 200000), rng.choice([16, 64, 100, 300, 301, 512, 768, 1024]),
                    rng.choice(["f32", "bf16"]), rng.random() < (0.3 if small else 0.7), rng.random() < 0.5,
                    rng.choice([0.0, 0.0, 0.1, 0.5]))


# ------------------------------------------------------------------------ inputs --

def _lengths(c):
    """The sets' lengths: a fixed draw of the case's range.  A causal set has no more queries than keys."""
    rng = random.Random("%d %d %d %d %d" % (c["sets"], c["q_lo"], c["q_hi"], c["k_lo"], c["k_hi"]))
    k = [rng.randint(c["k_lo"], c["k_hi"]) for _ in range(c["sets"])]
    if c["q_hi"] == 1 or c["cross"]:
        return [rng.randint(c["q_lo"], c["q_hi"]) for _ in range(c["sets"])], k
    return list(k), k


def _visible(c):
    """Pairs of a query and a key that it sees, over all sets."""
    total = 0
    for nq, nk in zip(*_lengths(c)):
        if not c["causal"]:
            total += nq * nk
            continue
        pre = min(c["prefix"], nk)
        lo = nk - nq + 1                       # keys that the first query sees without a prefix
        full = max(0, min(nq, pre - lo))       # queries whose own reach ends inside the prefix
        total += full * pre + sum(range(lo + full, nk + 1))
    return total


def _normal(g, *shape, dtype="f32", scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(TYPES[dtype])


def _unit_vectors(g, n, d):
    """Unit vectors with a decaying spectrum, as word embeddings have."""
    x = torch.randn(n, d, generator=g, device=DEV) * torch.arange(1, d + 1, device=DEV).float() ** -0.25
    return x / x.norm(dim=1, keepdim=True)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(c=c)
    if c["kind"] == "linear":
        dt = c["dtype"]
        s["x"] = _normal(g, c["rows"], c["d_in"], dtype=dt)
        s["w"] = _normal(g, c["d_out"], c["d_in"], dtype=dt, scale=c["d_in"] ** -0.5)
        s["b"] = _normal(g, c["d_out"], dtype=dt, scale=0.1) if c["bias"] else None
        s["r"] = _normal(g, c["rows"], c["d_out"], dtype=dt) if c["residual"] else None
        s["dy"] = _normal(g, c["rows"], c["d_out"], dtype=dt) if c["train"] else None
        return s
    if c["kind"] == "cross_entropy":
        w = _unit_vectors(g, c["vocab"], c["dim"])
        t = torch.randint(0, c["vocab"], (c["rows"],), generator=g, device=DEV)
        # early in training: the target is nearer than most words, but far from certain
        x = w[t] + 2.5 * c["dim"] ** -0.5 * torch.randn(c["rows"], c["dim"], generator=g, device=DEV)
        x = x / x.norm(dim=1, keepdim=True)
        left_out = torch.rand(c["rows"], generator=g, device=DEV) < c["ignored"]
        s["x"], s["w"] = x.to(TYPES[c["dtype"]]), w.to(TYPES[c["dtype"]])
        s["t"] = torch.where(left_out, torch.full_like(t, -1), t)
        s["b"] = 0.5 * torch.randn(c["vocab"], generator=g, device=DEV) if c["bias"] else None
        s["scale"] = 20.0                      # 1 / lambda at the embedding configurations' lambda = 0.05
        s["g"] = torch.rand(c["rows"], generator=g, device=DEV) / c["rows"] if c["train"] else None
        return s
    nq, nk = _lengths(c)
    h, hk, d, dt = c["heads"], c["kv_heads"], c["dim"], c["dtype"]
    s["q"] = _normal(g, sum(nq), h, d, dtype=dt)
    s["k"] = _normal(g, sum(nk), hk, d, dtype=dt)
    s["v"] = _normal(g, sum(nk), hk, d, dtype=dt)
    s["do"] = _normal(g, sum(nq), h, d, dtype=dt) if c["train"] else None
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, h + 1, device=DEV) / h)).float() if c["slopes"] else None
    s["prefix"] = torch.tensor([min(c["prefix"], k) for k in nk], dtype=torch.int32, device=DEV) if c["prefix"] else None
    lq, lk = torch.tensor(nq, device=DEV), torch.tensor(nk, device=DEV)
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    s["q_off"], s["k_off"] = torch.cat([zero, lq.cumsum(0)]), torch.cat([zero, lk.cumsum(0)])
    s["max_q"], s["max_k"] = max(nq), max(nk)
    # where each token stands in a batch padded to the longest set, and the token of each padded place
    for n, off, most, lens in (("q", s["q_off"], max(nq), lq), ("k", s["k_off"], max(nk), lk)):
        place = torch.arange(most, device=DEV)
        s[n + "_token"] = torch.minimum(off[:-1, None] + place, off[1:, None] - 1)
        of = torch.repeat_interleave(torch.arange(len(lens), device=DEV), lens)
        s[n + "_place"] = of * most + torch.arange(int(off[-1]), device=DEV) - off[of]
    return s


# ------------------------------------------------------------------- plain forms --

def _act(z, act):
    if act == "tanh":
        t = torch.tanh(z)
        return t, 1.0 - t * t
    if act == "relu":
        return torch.clamp(z, min=0.0), (z > 0).to(z.dtype)
    if act == "gelu":
        f = 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5))
        return z * f, f + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5
    if act == "silu":
        f = 1.0 / (1.0 + torch.exp(-z))
        return z * f, f * (1.0 + z * (1.0 - f))
    return z, torch.ones_like(z)


def _plain_linear(s):
    c, ty = s["c"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["b"] is not None:
        z = z + s["b"].float()
    y, slope = _act(z, c["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    out = dict(y=y.to(ty))
    if c["train"]:
        dz = s["dy"].float() * slope
        out["dx"], out["dw"] = (dz @ w).to(ty), (dz.t() @ x).to(ty)
        if s["b"] is not None:
            out["db"] = dz.sum(0).to(ty)
    return out


def _plain_entropy(s):
    ty = s["x"].dtype
    x, w, t = s["x"].float(), s["w"].float(), s["t"]
    z = s["scale"] * (x @ w.t())
    if s["b"] is not None:
        z = z + s["b"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    kept = t >= 0
    at = torch.clamp(t, min=0)
    loss = torch.where(kept, lse - z.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    out = dict(loss=loss, lse=lse)
    if s["g"] is not None:
        g = torch.where(kept, s["g"], torch.zeros_like(s["g"]))
        e = e * (g[:, None] / total)
        e.scatter_add_(1, at[:, None], -g[:, None])
        out["dx"], out["dw"] = (s["scale"] * (e @ w)).to(ty), (s["scale"] * (e.t() @ x)).to(ty)
        if s["b"] is not None:
            out["db"] = e.sum(0)
    return out


def _plain_attention(s):
    c, ty = s["c"], s["q"].dtype
    p, h, hk, d = c["sets"], c["heads"], c["kv_heads"], c["dim"]
    nq, nk, grp = s["max_q"], s["max_k"], c["heads"] // c["kv_heads"]

    def padded(x, token, of_keys):
        x = x.float()[token]                                               # set, place, head, dim
        if of_keys and grp > 1:
            x = x.repeat_interleave(grp, dim=2)
        return x.permute(0, 2, 1, 3).reshape(p * h, -1, d).contiguous()

    def tokens(x, place, heads):
        return x.view(p, heads, -1, d).permute(0, 2, 1, 3).reshape(-1, heads, d)[place].to(ty)

    q, k, v = padded(s["q"], s["q_token"], False), padded(s["k"], s["k_token"], True), padded(s["v"], s["k_token"], True)
    lq, lk = (s["q_off"][1:] - s["q_off"][:-1])[:, None, None], (s["k_off"][1:] - s["k_off"][:-1])[:, None, None]
    i, j = torch.arange(nq, device=DEV)[None, :, None], torch.arange(nk, device=DEV)[None, None, :]
    ahead = i + (lk - lq) - j                                              # how far the key lies behind the query
    seen = (j < lk) & (i < lq)
    if c["causal"]:
        reach = ahead >= 0
        if s["prefix"] is not None:
            reach = reach | (j < s["prefix"][:, None, None])
        seen = seen & reach
    z = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5
    z = z.view(p, h, nq, nk)
    slope = None
    if c["cap"] > 0:
        th = torch.tanh(z / c["cap"])
        z, slope = c["cap"] * th, 1.0 - th * th
    if s["slopes"] is not None:
        z = z - s["slopes"][None, :, None, None] * ahead.abs().float()[:, None]
    z = torch.where(seen[:, None], z, torch.full((), -math.inf, device=DEV))
    m = z.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(z - m)
    del z
    total = e.sum(3, keepdim=True)
    lse = (m + torch.log(total))[..., 0]                                   # set, head, place
    e = e / torch.where(total > 0, total, torch.ones_like(total))
    e = e.view(p * h, nq, nk)
    o = torch.bmm(e, v)
    out = dict(o=tokens(o, s["q_place"], h), lse=lse.permute(1, 0, 2).reshape(h, -1)[:, s["q_place"]])
    if c["train"]:
        do = padded(s["do"], s["q_token"], False)
        # places behind a set's end repeat its last token: they have no weight, since `seen` leaves them out
        ds = torch.bmm(do, v.transpose(1, 2).contiguous())
        ds = e * (ds - (do * o).sum(2, keepdim=True))
        if slope is not None:
            ds = ds * slope.view(p * h, nq, nk)
        ds = ds * d ** -0.5
        dv = torch.bmm(e.transpose(1, 2).contiguous(), do)
        del e
        dk = torch.bmm(ds.transpose(1, 2).contiguous(), q)
        out["dq"] = tokens(torch.bmm(ds, k), s["q_place"], h)
        out["dk"] = tokens(dk.view(p, hk, grp, nk, d).sum(2), s["k_place"], hk)
        out["dv"] = tokens(dv.view(p, hk, grp, nk, d).sum(2), s["k_place"], hk)
    return out


# --------------------------------------------------------------------- the library --

def _own_linear(s):
    import paper_2107_06876_amd as lcn
    c = s["c"]
    act = dict(none=lcn.ACT_NONE, tanh=lcn.ACT_TANH, relu=lcn.ACT_RELU, gelu=lcn.ACT_GELU, silu=lcn.ACT_SILU)[c["act"]]
    if not c["train"]:
        return dict(y=lcn.lcn_linear(s["x"], s["w"], bias=s["b"], residual=s["r"], activation=act))
    y, pre = lcn.lcn_linear(s["x"], s["w"], bias=s["b"], residual=s["r"], activation=act, keep_pre=True)
    dx, dw, db = lcn.lcn_linear_backward(s["x"], s["w"], pre, s["dy"], activation=act, with_bias=s["b"] is not None)
    out = dict(y=y, dx=dx, dw=dw)
    if db is not None:
        out["db"] = db
    return out


def _own_entropy(s):
    import paper_2107_06876_amd as lcn
    loss, lse = lcn.lcn_cross_entropy(s["x"], s["w"], s["t"], bias=s["b"], scale=s["scale"])
    out = dict(loss=loss, lse=lse)
    if s["g"] is not None:
        dx, dw, db = lcn.lcn_cross_entropy_backward(s["x"], s["w"], s["t"], lse, s["g"], bias=s["b"], scale=s["scale"])
        out["dx"], out["dw"] = dx, dw
        if db is not None:
            out["db"] = db
    return out


def _own_attention(s):
    import paper_2107_06876_amd as lcn
    c = s["c"]
    how = dict(causal=c["causal"], prefix=s["prefix"], slopes=s["slopes"], cap=c["cap"], max_q=s["max_q"])
    o, lse = lcn.lcn_attention(s["q"], s["k"], s["v"], s["q_off"], s["k_off"], **how)
    out = dict(o=o, lse=lse)
    if c["train"]:
        out["dq"], out["dk"], out["dv"] = lcn.lcn_attention_backward(s["q"], s["k"], s["v"], o, lse, s["do"], s["q_off"],
                                                                     s["k_off"], **how)
    return out


PLAIN = dict(linear=_plain_linear, attention=_plain_attention, cross_entropy=_plain_entropy)
OWN = dict(linear=_own_linear, attention=_own_attention, cross_entropy=_own_entropy)


def run(state):
    return (OWN if own else PLAIN)[state["c"]["kind"]](state)


def work(case):
    c = case
    e = SIZE[c["dtype"]]
    if c["kind"] == "linear":
        n, i, o = c["rows"], c["d_in"], c["d_out"]
        by = e * (n * i + i * o + n * o * (2 if c["residual"] else 1) + (o if c["bias"] else 0))
        if c["train"]:
            by += e * (n * o + n * i + i * o + (o if c["bias"] else 0))
        return dict(bytes=by, flops=2 * n * i * o * (3 if c["train"] else 1))
    if c["kind"] == "cross_entropy":
        n, v, d = c["rows"], c["vocab"], c["dim"]
        by = e * (n * d + v * d) + 8 * n + 8 * n + (4 * v if c["bias"] else 0)
        if c["train"]:
            by += e * (n * d + v * d) + 4 * n + (4 * v if c["bias"] else 0)
        return dict(bytes=by, flops=2 * n * v * d * (3 if c["train"] else 1))
    q, k = (sum(x) for x in _lengths(c))
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    by = e * d * (2 * q * h + 2 * k * hk) + 4 * q * h
    if c["train"]:
        by += e * d * (2 * q * h + 2 * k * hk)
    return dict(bytes=by, flops=_visible(c) * h * d * (14 if c["train"] else 4))


# ------------------------------------------------------------- results in 64 bits --

def _exact_linear(s):
    c = s["c"]
    x, w = s["x"].double(), s["w"].double()
    z = torch.addmm(s["b"].double(), x, w.t()) if s["b"] is not None else x.mm(w.t())
    z.requires_grad_(True)
    f = dict(none=lambda u: u * 1.0, tanh=torch.tanh, relu=torch.relu, gelu=torch.nn.functional.gelu,
             silu=torch.nn.functional.silu)[c["act"]]
    y = f(z)
    out = dict(y=(y if s["r"] is None else y + s["r"].double()).detach())
    if c["train"]:
        (dz,) = torch.autograd.grad(y, z, s["dy"].double())
        out["dx"], out["dw"] = dz.mm(w), dz.t().mm(x)
        if s["b"] is not None:
            out["db"] = dz.sum(0)
    return out


def _exact_entropy(s):
    c = s["c"]
    x, w, t = s["x"].double(), s["w"].double(), s["t"]
    loss, lse, dx = [], [], []
    dw, db = torch.zeros_like(w), torch.zeros(c["vocab"], dtype=torch.float64, device=DEV)
    step = max(1, 400_000_000 // c["vocab"])
    for a in range(0, c["rows"], step):
        xs, ts = x[a:a + step], t[a:a + step]
        z = s["scale"] * xs.mm(w.t())
        if s["b"] is not None:
            z += s["b"].double()
        n = torch.logsumexp(z, 1)
        rows = torch.nonzero(ts >= 0)[:, 0]
        l = torch.zeros_like(n)
        l[rows] = n[rows] - z[rows, ts[rows]]
        loss.append(l)
        lse.append(n)
        if c["train"]:
            gr = torch.zeros_like(n)
            gr[rows] = s["g"][a:a + step].double()[rows]
            gz = torch.exp(z - n[:, None]) * gr[:, None]
            gz[rows, ts[rows]] -= gr[rows]
            dx.append(s["scale"] * gz.mm(w))
            dw += s["scale"] * gz.t().mm(xs)
            db += gz.sum(0)
    out = dict(loss=torch.cat(loss), lse=torch.cat(lse))
    if c["train"]:
        out["dx"], out["dw"] = torch.cat(dx), dw
        if s["b"] is not None:
            out["db"] = db
    return out


def _exact_attention(s):
    c = s["c"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    do = s["do"].double() if c["train"] else None
    h, grp, d = c["heads"], c["heads"] // c["kv_heads"], c["dim"]
    o, lse = torch.zeros_like(q), torch.zeros(h, q.shape[0], dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    qo, ko = s["q_off"].tolist(), s["k_off"].tolist()
    pre = s["prefix"].tolist() if s["prefix"] is not None else [0] * c["sets"]
    for p in range(c["sets"]):
        a, b, e, f = qo[p], qo[p + 1], ko[p], ko[p + 1]
        rows = torch.arange(b - a, device=DEV)[:, None] + (f - e) - (b - a)
        cols = torch.arange(f - e, device=DEV)[None, :]
        hidden = (cols > rows) & (cols >= pre[p]) if c["causal"] else torch.zeros_like(cols > rows)
        far = (rows - cols).abs().double()
        step = h if (b - a) * (f - e) * h < 100_000_000 else 1             # all heads of a small set at once
        for x in range(0, h, step):
            hs, ks = list(range(x, x + step)), [y // grp for y in range(x, x + step)]
            Q, K, V = (u.permute(1, 0, 2).contiguous() for u in (q[a:b, hs], k[e:f, ks], v[e:f, ks]))
            z = torch.matmul(Q, K.transpose(1, 2).contiguous()) / math.sqrt(d)
            cut = 1.0
            if c["cap"] > 0:
                z = c["cap"] * torch.tanh(z / c["cap"])
                cut = 1.0 - (z / c["cap"]).square()
            if s["slopes"] is not None:
                z = z - s["slopes"][hs].double()[:, None, None] * far
            z = z.masked_fill(hidden, -math.inf)
            n = torch.logsumexp(z, 2)
            lse[hs, a:b] = n
            P = torch.exp(z - n[:, :, None])
            O = torch.matmul(P, V)
            o[a:b, hs] = O.permute(1, 0, 2)
            if c["train"]:
                D = do[a:b, hs].permute(1, 0, 2).contiguous()
                S = torch.matmul(D, V.transpose(1, 2).contiguous()) - (D * O).sum(2, keepdim=True)
                S = P * S * cut / math.sqrt(d)
                dq[a:b, hs] = torch.matmul(S, K).permute(1, 0, 2)
                gk = torch.matmul(S.transpose(1, 2).contiguous(), Q).permute(1, 0, 2)
                gv = torch.matmul(P.transpose(1, 2).contiguous(), D).permute(1, 0, 2)
                at = torch.tensor(ks, device=DEV)
                dk[e:f] = dk[e:f].index_add(1, at, gk)
                dv[e:f] = dv[e:f].index_add(1, at, gv)
    out = dict(o=o, lse=lse)
    if c["train"]:
        out.update(dq=dq, dk=dk, dv=dv)
    return out


def exact(case, seed):
    if work(case)["flops"] > 6e12:
        return None
    s = prepare(case, seed)
    return dict(linear=_exact_linear, attention=_exact_attention, cross_entropy=_exact_entropy)[case["kind"]](s)

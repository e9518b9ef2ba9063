"""What the tests of the encoder operators share: inputs, and how far results may be off.

Sums of K products in 32 bits whose terms have no common sign are off by about sqrt(K) roundings of 2^-24 of the
result; a bf16 output (8 significant bits) adds a rounding of at most 2^-8 of every value, an intermediate in bf16 (dz, G, P, dS) another of the
same size on terms that are then added.  All bounds are on the 2-norm of the difference over that of the result."""
import math

import torch

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def bound(dtype, k, intermediates=0):
    b = 2.0 ** -24 * (8 + 2 * math.sqrt(k))
    if dtype == BF16:
        b += 2.0 ** -8 * (1 + intermediates)
    return b


def off(got, want):
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    ok = torch.isfinite(want)
    norm = want[ok].norm().item()
    d = (got[ok] - want[ok]).norm().item()
    return d / norm if norm else d


def generator(*key):
    g = torch.Generator(device="cpu")
    seed = 17
    for k in key:
        seed = (seed * 1000003 + int(k)) % (1 << 31)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, scale=1.0, shift=0):
    """A contiguous device tensor; `shift` elements behind an aligned address."""
    n = math.prod(shape)
    flat = torch.zeros(n + shift, dtype=dtype, device=DEV)
    flat[shift:] = (scale * torch.randn(n, generator=g)).to(dtype).to(DEV)
    return flat[shift:].view(*shape)

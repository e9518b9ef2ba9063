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


# One rounding to bf16 by its statistics: half a unit in the last place is spread evenly, 2^-7 / sqrt(12) of the power of two below a
# value, which in the 2-norm over normally distributed ones is 0.734 to 0.737 of them, whatever their deviation (0.65 to 0.69 over
# values spread evenly, or evenly over octaves).  Independent roundings add in squares: two are 1.41 of one, so that a bound of 1.1
# tells one from two, and two from three.
ROUNDING = 0.737 * 2.0 ** -7 / math.sqrt(12.0)


def roundings(n):
    """The 2-norm of n independent roundings to bf16, with a tenth of room."""
    return 1.1 * ROUNDING * math.sqrt(n)


def farthest(got, want):
    """The largest error of a value of bf16 tensors over what it may be: 2^-8 of the value (its own rounding) and 2^-6.5 of the root
    mean square of its row (last dimension): 7 deviations of a sum whose terms were each rounded once."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape and torch.isfinite(got).all()
    row = want.square().mean(-1, keepdim=True).sqrt()
    return ((got - want).abs() / (2.0 ** -8 * want.abs() + 2.0 ** -6.5 * row + 1e-30)).max().item()

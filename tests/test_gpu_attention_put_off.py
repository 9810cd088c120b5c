"""Tiles whose hidden keys hold an infinity or NaN: the seen keys beside them keep one
weight, in the sum of the weights as in the sum of the values, whatever their scores."""
import math

import pytest
import torch

from tests._cache import U, Batch
from tests._exact import Exact, largest_step
from tests.test_gpu_paged_attention import run

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "f16", "f32"]


def spoil(b, at, bad):
    page, off = b.where(0, at)
    b.v[page, :, off] = bad


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("size", [2.0 ** 0, 2.0 ** 5, 2.0 ** 8, 2.0 ** 10])
@pytest.mark.parametrize("dim", [64, 128])
def test_one_key_stands_out(dim, size, dt):
    """Its score (up to dim 2^20, no short number) is far above the others: the output is
    its value.  u for the output, 4 roundings of 2^-24 in fp32 (weight times value, the
    sum's reciprocal, its product, the others' weights: 0).  In a tile that is not put off
    (position 2000) its weight is an operand of a 16-bit product: the running maximum may
    lag, so that it is some w in [1, 2^8], rounded to w (1 + d), |d| <= u, while the sum of
    weights is w: out = v (1 + d) (1 + e), |e| <= u, off by at most 2 u + u^2."""
    for keys, first, bad, at in ((200, 70, [66], 100), (200, 70, [66], 199), (128, 3, [0], 40),
                                 (3000, 130, [128, 129], 131), (3000, 130, [128], 2000)):
        b = Batch([1], [keys], 4, 2, dim, 16, dt, seed=keys + at)
        page, off = b.where(0, [at])
        b.q[:] = (b.q * size).to(b.q.dtype)
        b.q[:, 1::2] = b.q[:, ::2]            # (the heads that share a key: one query)
        b.k[page, :, off] = (b.q[:, ::2] * 2).to(b.k.dtype)
        spoil(b, bad, math.nan)
        got = run(b, dict(scale=1.0), first=[first])[0].double().cpu()
        v = b.v[page, :, off][0].double().repeat_interleave(2, 0)
        u = U[dt] if dt != "f32" else 0.0
        tol = (2 * u + u * u if at == 2000 else u) * v.abs() + 4 * 2.0 ** -24 * v.abs() + 1e-6 * U[dt]
        assert ((got - v).abs() <= tol).all(), (keys, at, float((got / v).min()), float((got / v).max()))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("exponent", [8, 17, 22, 23, 25, 26])
@pytest.mark.parametrize("keys,heads,dim", [(640, 2, 64), (640, 1024, 8), (3000, 2, 64)])
def test_exact_scores_beside_bad_values(keys, heads, dim, exponent, dt):
    """Keys of like scores in tiles that are put off and in others, in one range and in
    several; rising and falling."""
    step = largest_step(exponent)
    for order in ((0, 1, 3, 2, 1), (9, 1, 0, 1, 3), (0, 3, 7, 13, 18), (18, 12, 6, 2, 0)):
        at = (70, 71, 127, 300, keys - 1)
        b = Exact(keys, heads, dim, 16, dt, {a: (exponent, step * d) for a, d in zip(at, order)})
        spoil(b, [3, 66], math.nan)
        spoil(b, [67], -math.inf)
        b.compare(run(b, dict(scale=1.0), first=[70]), torch.arange(keys) >= 70)


@pytest.mark.parametrize("dt", TYPES)
def test_more_than_64_such_tiles(dt):
    """Two rows of a wave: bad values hidden from one, in 90 tiles of one range."""
    keys = 6000
    b = Exact(keys, 1024, 8, 16, dt, {5500: (17, 0), 5990: (17, 1), 5998: (17, 2)})
    two = Batch([2], [keys], 1024, 1024, 8, 16, dt, seed=1, fill=0.0)
    two.q[:], two.table, two.pages, two.k, two.v = b.q[0], b.table, b.pages, b.k, b.v
    spoil(two, list(range(3, 5400, 40)), math.nan)
    got = run(two, dict(scale=1.0), first=[0, 5450])
    b.compare(got[1:], torch.arange(keys) >= 5450)


@pytest.mark.parametrize("dt", TYPES)
def test_missing_page_and_a_bad_first_row(dt):
    """Pages that are none are read as the cache's first row, which holds NaN."""
    b = Exact(400, 2, 64, 16, dt, {40: (17, 0), 70: (17, 1), 390: (17, 2)})
    b.table[b.table == 0] = b.pages          # (the cache's first page moves behind the others)
    for name in ("k", "v"):
        old = getattr(b, name)
        setattr(b, name, torch.cat([old, old[:1]]))
    b.pages += 1
    b.k[0], b.v[0] = math.nan, math.nan
    seen = torch.ones(400, dtype=torch.bool)
    for p in (5, 20):
        b.table[0, p] = -1
        seen[16 * p:16 * p + 16] = False
    got = run(b, dict(scale=1.0))
    b.table[0, 5], b.table[0, 20] = 1, 1     # (any page: the values there are not seen)
    b.compare(got, seen)

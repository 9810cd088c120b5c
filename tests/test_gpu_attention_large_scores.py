"""Scores that are exact in fp32, however large, weigh by their differences: the same
softmax whether two keys meet in one tile, in one range or in the join."""
import pytest
import torch

from tests._exact import Exact, largest_step
from tests.test_gpu_paged_attention import run

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "f16", "f32"]
EXPONENTS = [8, 17, 20, 21, 22, 23, 24, 25, 26]
ORDERS = [(0, 1, 3, 2, 1), (9, 1, 0, 1, 3), (0, 0, 0, 0, 0), (0, 3, 7, 13, 18), (18, 12, 6, 2, 0)]


def scores(at, order, exponent):
    step = largest_step(exponent)
    return {a: (exponent, step * d) for a, d in zip(at, order)}


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("exponent", EXPONENTS)
def test_keys_in_different_ranges(exponent, dt):
    for order in ORDERS:
        b = Exact(3000, 2, 64, 16, dt, scores((10, 700, 1400, 2100, 2990), order, exponent))
        b.compare(run(b, dict(scale=1.0)))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("exponent", EXPONENTS)
def test_keys_in_one_range(exponent, dt):
    """So many heads that a row's ten tiles are one range: its maximum rises on the way."""
    for order in ORDERS:
        b = Exact(640, 1024, 8, 16, dt, scores((10, 130, 320, 400, 630), order, exponent))
        b.compare(run(b, dict(scale=1.0)))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("exponent", EXPONENTS)
def test_keys_in_one_tile(exponent, dt):
    for order in ORDERS:
        b = Exact(64, 2, 64, 16, dt, scores((1, 30, 31, 32, 63), order, exponent))
        b.compare(run(b, dict(scale=1.0)))


@pytest.mark.parametrize("dt", TYPES)
def test_scales(dt):
    """The same scores with a scale: 2^25 of a product of 2^37, and of one of 2^13."""
    for exponent, scale in ((25, 2.0 ** -6), (13, 2.0 ** 12)):
        b = Exact(3000, 2, 64, 16, dt, scores((10, 700, 1400, 2100, 2990), (0, 1, 3, 2, 1), exponent))
        b.scores = b.scores * scale
        b.compare(run(b, dict(scale=scale)))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("keys,heads,dim", [(200, 2, 64), (3000, 2, 64), (640, 1024, 8)])
def test_products_whose_scores_pass_fp32(keys, heads, dim, dt):
    """Products of 2^68 and more with a scale of 2^60, of either sign: the largest alone
    (the others' weights are e^-(2^100))."""
    for sign in (1.0, -1.0):
        for best in (0, keys // 2, keys - 1):
            b = Exact(keys, heads, dim, 16, dt, {0: (2, 1)})
            b.q[:, :, 0], b.q[:, :, 1] = 2.0 ** 34, 0.0
            k = torch.zeros(keys, heads, dim)
            k[:, :, 0] = sign * 2.0 ** (36 if sign < 0 else 34)
            k[best, :, 0] = sign * 2.0 ** (34 if sign < 0 else 36)
            b.put(b.k, 0, k)
            got = run(b, dict(scale=2.0 ** 60))[0].cpu()
            want = b.get(b.v, 0)[best].double()
            # (the weight is 1, or 2^7 in fp32 sums of products: exact but for 3 roundings of 2^-24)
            assert ((got.double() - want).abs() <= 4 * 2.0 ** -24 * want.abs()).all(), (sign, best)

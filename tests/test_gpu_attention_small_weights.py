"""A long flat tail beside one strong key: fp16 weights far below the strong key's keep
their part of the sum."""
import math

import pytest
import torch

from tests._cache import U, Batch
from tests.test_gpu_paged_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("below", [12, 16, 20, 24, 26, 28, 30])
@pytest.mark.parametrize("keys,heads", [(60000, 2), (6000, 256)])
def test_flat_tail(keys, heads, below, dt):
    """Values of 0 at the strong key and 1024 elsewhere, whose weights are 2^-below of the
    strong one's.  Bound: an fp16 weight is an operand of at most half a step below its
    type's range (2^-25), 2^7 above its size relative to the largest: 2^-32 a key; u for a
    weight and for the output; scores (one product of short numbers) and exponentials 2^-20
    of the weight; sums of n terms n + 64 roundings of 2^-24."""
    b = Batch([1], [keys], heads, heads, 8, 64, dt, seed=below)
    b.q[:] = 0.0
    b.q[:, :, 0] = 1.0
    k, v = torch.zeros(keys, heads, 8), torch.full((keys, heads, 8), 1024.0)
    strong = keys // 3
    k[strong, :, 0], v[strong] = float(below), 0.0
    b.put(b.k, 0, k)
    b.put(b.v, 0, v)
    got = run(b, dict(scale=math.log(2.0)))[0].double().cpu()
    # (the scale is rounded to fp32: 2^-24 of an exponent of 30 at most)
    tail = (keys - 1) * 2.0 ** -below
    want = 1024.0 * tail / (1.0 + tail)
    u, lost = {"bf16": (U["bf16"], 0.0), "f16": (U["f16"], 2.0 ** -32), "f32": (0.0, 0.0)}[dt]
    tol = 1024.0 * keys * lost + (2 * u + 2.0 ** -18 + (keys + 64) * 2.0 ** -24) * want
    assert ((got - want).abs() <= tol).all(), (float(got.min()), float(got.max()), want, tol)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_weights_above_the_running_maximum(dim):
    """fp16 scores that rise by just less than what makes the maximum follow (2^8), near
    every size where the products round: no weight passes the type's largest number."""
    for exponent in (4, 10, 20, 21, 22, 23):
        step = max(1.0, 2.0 ** (exponent - 23))
        low = exponent // 2
        for rise in (5.0, 5.5, 6.0):
            b = Batch([1], [640], 1024, 1024, 8, 16, "f16", seed=1) if dim == 64 else \
                Batch([40], [640], 2, 2, dim, 16, "f16", seed=1)
            b.q[:] = 0.0
            b.q[:, :, 0], b.q[:, :, 1] = 2.0 ** low, 1.0
            k = torch.zeros(640, b.kv_heads, b.dim)
            k[:, :, 0] = 2.0 ** (exponent - low)
            k[:, :, 1] = (step * torch.round(torch.arange(640) // 64 * rise / step))[:, None]
            b.put(b.k, 0, k)
            v = b.get(b.v, 0).double()
            got = run(b, dict(scale=1.0, causal=False)).double().cpu()
            w = torch.softmax(k[:, 0, 1].double(), 0)
            want, size = (w[:, None, None] * v).sum(0), (w[:, None, None] * v.abs()).sum(0)
            tol = (2 * U["f16"] + 2.0 ** -14) * size + 640 * 2.0 ** -25
            assert ((got - want).abs() <= tol).all(), (exponent, rise)

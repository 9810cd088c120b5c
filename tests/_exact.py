"""Batches of one row a request whose scores are given whole numbers, exact in fp32 and in
any order of the sum: q = (2^a, 1, 0 ...), k = (2^b, d, 0 ...), score 2^(a + b) + d, or 0
where k is 0.  Their softmax in 64 bits follows from the differences alone."""
import math

import torch

from tests._cache import U, Batch


class Exact(Batch):
    """Request 0 alone: scores[position] = (exponent, d); all other keys score 0."""

    def __init__(self, keys, heads, dim, page, dt, scores, seed=0):
        super().__init__([1], [keys], heads, heads, dim, page, dt, seed=seed, fill=0.0)
        self.q[:] = 0.0
        exponent = {e for e, _ in scores.values()}.pop()
        low = exponent // 2
        self.q[:, :, 0], self.q[:, :, 1] = 2.0 ** low, 1.0
        k = torch.zeros(keys, heads, dim)
        for at, (e, d) in scores.items():
            k[at, :, 0], k[at, :, 1] = 2.0 ** (e - low), d
        self.put(self.k, 0, k)
        assert torch.equal(self.get(self.k, 0).float(), k)
        x = torch.zeros(keys, dtype=torch.float64)
        for at, (e, d) in scores.items():
            x[at] = 2.0 ** e + d
        self.scores = x

    def expected(self, seen=None):
        """(out, bound) [heads, dim] in 64 bits.  A weight's exponent is a difference of
        exact scores: it is off by the roundings of the difference times log2(e), 2^-24 of
        at most 2^8 each where the weight is not below 2^-126, and by the exponential's
        two steps, on both sides of a factor between ranges: 2^-14 in all.  16-bit types
        round weight and output by u each."""
        x, v = self.scores, self.get(self.v, 0).double()
        if seen is not None:
            x, v = x[seen], v[seen]
        w = torch.exp(x - x.max())
        w = w / w.sum()
        y, size = (w[:, None, None] * v).sum(0), (w[:, None, None] * v.abs()).sum(0)
        u = 0.0 if self.dt == "f32" else U[self.dt]
        return y, (2 * u + 2.0 ** -14) * size + 1e-6

    def compare(self, got, seen=None):
        y, err = self.expected(seen)
        bad = ~((got[0].double().cpu() - y).abs() <= err)
        assert not bad.any(), (int(bad.sum()), float(got[0].cpu()[bad][0]), float(y[bad][0]))


def largest_step(exponent):
    """The step between neighbouring fp32 numbers from 2^exponent on, 1 at least."""
    return max(1.0, 2.0 ** (exponent - 23))

"""Batches over a paged cache for the attention tests, and the operators'
formulas in 64 bits (torch on the CPU; no code of the package)."""
import math

import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# half a step of a rounding, relative to the value; half a step below the normal range
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -134, "f16": 2.0 ** -25, "f32": 2.0 ** -150}


class Batch:
    """Requests of rows[r] rows and keys[r] keys, their pages anywhere in a cache whose
    other rows hold NaN; `spare` rows behind the last request."""

    def __init__(self, rows, keys, heads, kv_heads, dim, page, dt, seed=0, spare=0, table_pages=None,
                 fill=float("nan")):
        g = torch.Generator().manual_seed(7000 + seed)
        self.rows, self.keys, self.page = list(rows), list(keys), page
        self.heads, self.kv_heads, self.dim, self.dt = heads, kv_heads, dim, dt
        per = [-(-k // page) for k in keys]
        self.table_pages = table_pages or max(1, max(per))
        self.pages = sum(per) + 2
        order = torch.randperm(self.pages, generator=g).to(torch.int32)
        self.table = torch.full((len(rows), self.table_pages), -7, dtype=torch.int32)
        at = 0
        for r, p in enumerate(per):
            self.table[r, :p] = order[at:at + p]
            at += p
        self.start = [0] + list(np.cumsum(rows))
        self.tokens = self.start[-1] + spare
        shape = (self.pages, kv_heads, page, dim)
        self.k = torch.full(shape, fill).to(DT[dt])
        self.v = torch.full(shape, fill).to(DT[dt])
        for r in range(len(rows)):
            for cache in (self.k, self.v):
                self.put(cache, r, torch.randn(keys[r], kv_heads, dim, generator=g))
        self.q = (2.0 * torch.randn(self.tokens, heads, dim, generator=g)).to(DT[dt])
        self.g = g

    def where(self, r, positions):
        p = torch.as_tensor(positions, dtype=torch.int64)
        return self.table[r].long()[p // self.page], p % self.page

    def put(self, cache, r, values, at=0):
        """values [n, kv_heads, dim] to request r's positions from `at`."""
        page, off = self.where(r, torch.arange(at, at + values.shape[0]))
        cache[page, :, off] = values.to(cache.dtype)

    def get(self, cache, r, n=None):
        page, off = self.where(r, torch.arange(self.keys[r] if n is None else n))
        return cache[page, :, off]

    def ints(self, v):
        return torch.as_tensor(v, dtype=torch.int32).cuda()

    def gpu(self):
        """q_start, kv_len, page_table on the GPU."""
        return self.ints(self.start), self.ints(self.keys), self.table.cuda()

    def desc(self, abi, **kw):
        kw = dict(dict(max_queries=max(max(self.rows), 1), max_keys=max(max(self.keys), 1)), **kw)
        return abi.kv_desc(self.tokens, len(self.rows), self.heads, self.kv_heads, self.dim,
                           self.pages, self.page, self.table_pages, DT[self.dt], **kw)


def softmax_rows(x, sees, v):
    """x, sees [rows, keys], v [keys, dim] -> (out, sum of w |v|, number of seen keys' |v|)"""
    x = torch.where(sees, x, -math.inf)
    top = x.amax(1, keepdim=True)
    p = torch.where(sees, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
    total = p.sum(1, keepdim=True)
    w = torch.where(total > 0, p / total, 0.0)
    if torch.isfinite(v).all():
        return w, w @ v, w @ v.abs(), sees.double() @ v.abs()
    own = torch.where(sees[:, :, None], v, 0.0)      # [rows, keys, dim]
    w3 = w[:, :, None]
    return w, (w3 * own).sum(1), (w3 * own.abs()).sum(1), own.abs().sum(1)


def attention(b, sees_of, far_of, scale, cap=0.0, slopes=None, skip=()):
    """(out, error bound) [tokens, heads, dim]; rows of no request: NaN and infinity.

    Bound: a score is off by dim + 16 roundings of 2^-24 of sum |q k| scale, and by
    16 of them of itself, the cap (at most 256 of it: above, 64 of itself) and the bias; twice that is a weight's relative error
    (its own and the sum's).  Weights are rounded to the type (u, and half a step below
    its normal range, 2^8 of it at most since the running maximum may lag by 2^8 - the
    sum is at least 1), sums of n terms take n + 64 roundings of 2^-24, the output u."""
    u, tiny = U[b.dt], TINY[b.dt]
    out = torch.full((b.tokens, b.heads, b.dim), math.nan, dtype=torch.float64)
    err = torch.full_like(out, math.inf)
    group = b.heads // b.kv_heads
    for r, n in enumerate(b.rows):
        if not n or r in skip:
            continue
        mine = slice(b.start[r], b.start[r] + n)
        sees, far = sees_of(r), far_of(r)
        k, v = b.get(b.k, r).double(), b.get(b.v, r).double()
        for h in range(b.heads):
            q, kh, vh = b.q[mine, h].double(), k[:, h // group], v[:, h // group]
            clean = torch.where(sees.any(0)[:, None], kh, 0.0)
            x = q @ clean.t() * scale
            size = q.abs() @ clean.abs().t() * scale
            off = (b.dim + 16) * 2.0 ** -24 * size + 2.0 ** -20 * x.abs()
            if cap:
                x = cap * torch.tanh(x / cap)
                off = off + (2.0 ** -20 * cap if cap <= 256 else 2.0 ** -18 * x.abs())
            if slopes is not None:
                x = x - float(slopes[h]) * far
                off = off + 2.0 ** -20 * (float(slopes[h]) * far).abs()
            off = torch.where(sees, off, 0.0).amax(1, keepdim=True)
            w, y, size, all_v = softmax_rows(x, sees, vh)
            rel = torch.expm1(2 * off) + (sees.sum(1, keepdim=True) + 64) * 2.0 ** -24
            out[mine, h] = y
            err[mine, h] = ((rel + (u if b.dt != "f32" else 0.0)) * size + u * y.abs() * (1 + rel) +
                            tiny * all_v + tiny + 1e-37)
    return out, err


def check(got, ref, err, what):
    got = got.double().cpu()
    bad = ~((got - ref).abs() <= err) & torch.isfinite(err)
    assert not bad.any(), (what, int(bad.sum()), [int(i) for i in bad.nonzero()[0]],
                           float(got[bad][0]), float(ref[bad][0]), float(err[bad][0]))

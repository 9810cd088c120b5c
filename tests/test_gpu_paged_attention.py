"""sparoa_paged_attention against its formula in 64 bits (tests/_cache.py, where the
tolerance is derived): lengths from one key to many tiles, shared heads, head sizes
that fill no tile, pages of every size, masks that leave a row empty, infinities
and NaN in hidden places, batches that break their bounds."""
import math

import pytest
import torch

from tests._cache import DT, Batch, attention, check

pytestmark = pytest.mark.gpu


def _abi():
    from paper_2511_19457_amd import abi
    return abi


def run(b, opts=None, prefix=None, first=None, slopes=None, out=None, stream=None, ws_fill=255,
        **desc):
    abi = _abi()
    d = b.desc(abi, **desc)
    o = abi.attention_opts(**dict(dict(scale=b.dim ** -0.5), **(opts or {})))
    ws = torch.full((max(16, abi.sparoa_attention_workspace_size(d)),), ws_fill,
                    dtype=torch.uint8, device="cuda")
    if out is None:
        out = torch.full((b.tokens, b.heads, b.dim), 7.0, dtype=DT[b.dt], device="cuda")
    abi.sparoa_paged_attention(d, o, b.q.cuda(), b.k.cuda(), b.v.cuda(), *b.gpu(),
                               None if prefix is None else b.ints(prefix),
                               None if first is None else b.ints(first),
                               None if slopes is None else slopes.float().cuda(), out, ws, stream)
    torch.cuda.synchronize()
    return out


def visible(b, r, causal=True, window=0, prefix=None, first=None, pageless=None):
    n, length = b.rows[r], b.keys[r]
    p = torch.arange(length - n, length)[:, None]
    k = torch.arange(length)[None]
    s = torch.ones(n, length, dtype=torch.bool)
    if causal:
        s = k <= (p if prefix is None else torch.maximum(p, torch.tensor(prefix[r] - 1)))
    if window:
        s = s & (k > p - window)
    if first is not None:
        s = s & (k >= torch.as_tensor(first[b.start[r]:b.start[r] + n])[:, None])
    if pageless is not None and r in pageless:
        s = s & ~torch.isin(k // b.page, torch.tensor(pageless[r]))
    return s


def distance(b, r):
    n, length = b.rows[r], b.keys[r]
    return (torch.arange(length - n, length)[:, None] - torch.arange(length)[None]).abs().double()


def compare(b, opts=None, prefix=None, first=None, slopes=None, pageless=None, skip=(), **desc):
    o = dict(dict(causal=True, window=0, cap=0.0, scale=b.dim ** -0.5), **(opts or {}))
    got = run(b, opts, prefix, first, slopes, **desc)
    ref, err = attention(
        b, lambda r: visible(b, r, o["causal"], o["window"], prefix, first, pageless),
        lambda r: distance(b, r), o["scale"], o["cap"], slopes, skip)
    check(got, ref, err, (b.dt, b.rows, b.keys, b.dim, opts))
    untouched = torch.isinf(err).all(2).all(1)
    assert (got.cpu()[untouched] == 7.0).all()
    return got


TYPES = ["bf16", "f16", "f32"]
SHAPES = [
    # rows, keys, heads, kv_heads, dim, page
    ([1], [1], 1, 1, 64, 16),
    ([1], [63], 4, 4, 64, 16),
    ([1], [64], 8, 1, 128, 1),
    ([1], [65], 8, 2, 128, 64),
    ([1], [1500], 32, 8, 128, 16),
    ([1, 1, 1, 1, 1], [5, 700, 33, 1, 129], 12, 3, 80, 25),
    ([3, 1, 0, 40], [3, 200, 0, 77], 5, 1, 128, 7),
    ([130], [130], 2, 2, 64, 32),
    ([65, 200], [65, 333], 4, 2, 128, 16),
    ([33, 7], [500, 7], 3, 3, 40, 16),
    ([50], [190], 6, 2, 192, 24),
    ([20, 1], [150, 90], 4, 2, 256, 16),
    ([9], [2100], 2, 1, 8, 100),
]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,keys,heads,kv,dim,page", SHAPES)
def test_causal(rows, keys, heads, kv, dim, page, dt):
    compare(Batch(rows, keys, heads, kv, dim, page, dt, seed=len(rows) + dim, spare=3))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("opts", [dict(causal=False), dict(window=1), dict(window=64),
                                  dict(window=100, causal=False), dict(cap=5.0),
                                  dict(cap=30.0, window=37), dict(scale=0.5),
                                  dict(window=410), dict(window=411), dict(window=2 ** 31 - 2),
                                  dict(window=2 ** 40)])
def test_options(opts, dt):
    compare(Batch([70, 1, 150], [70, 300, 411], 4, 2, 64, 20, dt, seed=5), opts)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("cap", [2.0 ** -60, 1e-3, 256.0, 257.0, 1e4, 1e6, 2.0 ** 60])
def test_caps_of_any_size(cap, dt):
    """A cap far above the scores changes nothing in them; a tiny one leaves equal weights."""
    b = Batch([40, 1], [100, 300], 4, 2, 64, 16, dt, seed=8)
    compare(b, dict(cap=cap))
    compare(b, dict(cap=cap, scale=20.0))
    compare(b, dict(cap=cap), slopes=2.0 ** -torch.arange(1.0, 5.0))


def test_least_scale():
    """All visible keys alike; with slopes, as their distances alone."""
    b = Batch([1], [200], 2, 2, 64, 16, "f32", seed=9)
    compare(b, dict(scale=2.0 ** -60))
    compare(b, dict(scale=2.0 ** -60), slopes=torch.tensor([0.5, 0.25]))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("keys", [1, 200, 3000])
@pytest.mark.parametrize("scale,size", [(2.0 ** 60, 1.0), (1.0, 2.0 ** 15), (2.0 ** 40, 2.0 ** 15)])
def test_scores_far_above_one(scale, size, keys, dt):
    """The best key alone: one that stands out, or the last of rising ones, which an eighth
    of a step or more parts from the next (their products are exact)."""
    b = Batch([1], [keys], 2, 2, 64, 16, dt, seed=9)
    sign = torch.sign(b.q[0].float())
    b.q[0] = (size * sign).to(b.q.dtype)
    for rising in (False, True):
        k = torch.zeros(keys, 2, 64)
        if rising:
            k[:] = size * sign * (torch.arange(keys) * 16 // keys / 16 - 0.5)[:, None, None]
            k[-1] = size * sign
        else:
            k[keys // 3] = size * sign
        b.put(b.k, 0, k)
        best = keys - 1 if rising else keys // 3
        assert torch.equal(run(b, dict(scale=scale))[0].cpu(), b.get(b.v, 0)[best])


@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("keys", [2, 31, 32, 33, 63, 64, 65, 96, 128, 129, 200])
def test_windows_within_few_tiles(keys, dim):
    """Windows shorter than the cache, caches of one tile or a few, bounds that just hold."""
    for rows in (1, 2, min(keys, 40)):
        for window in (1, 10, 31, 33, 63, 100):
            compare(Batch([rows], [keys], 4, 1, dim, 16, "f32", seed=keys), dict(window=window))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("opts", [{}, dict(cap=10.0), dict(window=90), dict(causal=False)])
def test_prefix_documents_slopes(opts, dt):
    b = Batch([70, 1, 150], [70, 300, 411], 6, 3, 80, 16, dt, seed=6, spare=2)
    p = torch.cat([torch.arange(k - n, k) for n, k in zip(b.rows, b.keys)] + [torch.zeros(2)])
    first = (p - p % 33).int().tolist()
    slopes = 2.0 ** -torch.arange(1.0, 7.0)
    compare(b, opts, prefix=[50, 0, 1000])
    compare(b, opts, first=first)
    compare(b, opts, prefix=[64, 400, 300], first=first, slopes=slopes)


@pytest.mark.parametrize("dt", TYPES)
def test_rows_that_see_nothing(dt):
    """first_key behind a row's own key: zeros, beside rows that see some."""
    b = Batch([40, 1], [100, 9], 4, 2, 64, 16, dt, seed=7)
    first = [0, 1000, 61] * 13 + [99] + [9]
    got = compare(b, first=first)
    assert (got[1] == 0).all() and (got[40] == 0).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_hidden_infinities(bad, dim, dt):
    """Rows before a bad value's position do not meet it."""
    b = Batch([80], [150], 4, 2, dim, 16, dt, seed=8)
    for at in (101, 149):
        page, off = b.where(0, [at])
        b.v[page, 1, off, 3] = bad
        b.k[page, 0, off, 5] = bad
    got = run(b).double().cpu()
    ref, err = attention(b, lambda r: visible(b, r), lambda r: distance(b, r), dim ** -0.5)
    ok = torch.ones(80, 4, dim, dtype=torch.bool)
    ok[31:] = False                       # (row 31 is the first to see position 101)
    check(torch.where(ok, got, 0.0), torch.where(ok, ref, 0.0), torch.where(ok, err, 1.0), bad)
    assert torch.isfinite(got[:31]).all()
    # heads 2 and 3 read the bad value: that dimension, and no other, is bad from there on
    assert not torch.isfinite(got[31:, 2:, 3]).any()
    others = [d for d in range(dim) if d != 3]
    assert torch.isfinite(got[31:, 2:, others]).all()
    check(got[31:, 2:, others], ref[31:, 2:, others], err[31:, 2:, others], bad)


@pytest.mark.parametrize("dt", TYPES)
def test_hidden_infinities_in_every_tile(dt):
    """A document that begins late, behind bad values in tiles of the other row's: few
    ranges (many heads), so that one work-group meets more than 64 such tiles."""
    b = Batch([2], [6000], 1024, 1024, 8, 16, dt, seed=18)
    for at in range(3, 5400, 40):
        page, off = b.where(0, [at])
        b.v[page, :, off, 1] = math.nan if at % 3 else math.inf
    first = [0, 5450]
    got = run(b, first=first).double().cpu()
    sees, u = visible(b, 0, first=first)[1:], {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 0.0}[dt]
    assert torch.isfinite(got[1]).all()
    for h in (0, 1, 500, 1023):
        k, v = b.get(b.k, 0)[:, h].double(), b.get(b.v, 0)[:, h].double()
        k, v = k[sees[0]], v[sees[0]]
        x = (b.q[1:, h].double() @ k.t()) * 8 ** -0.5
        w = torch.softmax(x, 1)
        # weights and the output are rounded (u each), scores off by 24 roundings of 2^-24
        size = w @ v.abs()
        off = torch.expm1(2 * 24 * 2.0 ** -24 * (b.q[1:, h].double().abs() @ k.abs().t()).max() +
                          2.0 ** -19 * x.abs().max())
        assert ((got[1, h] - w @ v).abs() <= (2 * u + off + 700 * 2.0 ** -24) * size + 1e-4 * u).all()


@pytest.mark.parametrize("dt", TYPES)
def test_large_scores(dt):
    """Scores of hundreds, and a maximum that keeps rising."""
    b = Batch([30, 1], [400, 1000], 2, 1, 64, 16, dt, seed=9)
    for r in range(2):
        k = b.get(b.k, r).double()
        b.put(b.k, r, k * torch.linspace(0.1, 6, k.shape[0])[:, None, None].double())
    compare(b, dict(scale=1.0))


def test_weights_below_the_first_tile():
    """All weight on one key, wherever it lies."""
    for at in (0, 5, 63, 64, 200, 639):
        b = Batch([1], [640], 2, 2, 64, 16, "bf16", seed=10)
        k = torch.zeros(640, 2, 64)
        k[at] = b.q[0].float() * 10
        b.put(b.k, 0, k)
        got = run(b, dict(scale=1.0))
        assert torch.equal(got[0].cpu(), b.get(b.v, 0)[at])


@pytest.mark.parametrize("dt", TYPES)
def test_pages_that_are_none(dt):
    b = Batch([6, 1, 90], [100, 333, 400], 4, 2, 128, 16, dt, seed=11)
    lost = {0: [2], 1: [0, 20], 2: [1, 2, 3, 4, 22]}
    bad = [-1, b.pages, 2 ** 31 - 1, -2 ** 31, b.pages + 1]
    ref = Batch([6, 1, 90], [100, 333, 400], 4, 2, 128, 16, dt, seed=11)
    for r, pages in lost.items():
        for i, p in enumerate(pages):
            b.table[r, p] = bad[i]
    got = run(b)
    want, err = attention(ref, lambda r: visible(ref, r, pageless=lost),
                          lambda r: distance(ref, r), 128 ** -0.5)
    check(got, want, err, "pages")


@pytest.mark.parametrize("dt", TYPES)
def test_requests_out_of_bounds_are_left_out(dt):
    b = Batch([4, 5, 6, 2], [40, 50, 60, 20], 2, 1, 64, 16, dt, seed=12)
    # more rows than max_queries, more keys than max_keys
    compare(b, skip=(2,), max_queries=5)
    compare(b, skip=(2,), max_keys=59)
    # fewer keys than rows, rows before 0, backwards, past the end
    q_start, kv_len, table = b.gpu()
    abi = _abi()
    d = b.desc(abi)
    ws = torch.empty(max(16, abi.sparoa_attention_workspace_size(d)), dtype=torch.uint8,
                     device="cuda")
    ref, err = attention(b, lambda r: visible(b, r), lambda r: distance(b, r), 64 ** -0.5)
    for starts, lens, gone in (([0, 4, 9, 15, 17], [3, 50, 60, 20], (0, 4)),
                               ([-3, 4, 9, 15, 17], [40, 50, 60, 20], (0, 4)),
                               ([0, 4, 9, 15, 99], [40, 50, 60, 20], (15, 17)),
                               ([0, 4, 9, 8, 17], [40, 50, 60, 20], (9, 17)),
                               ([0, 4, 9, 15, 17], [40, -5, 60, 2 ** 30], (4, 9))):
        out = torch.full((17, 2, 64), 7.0, dtype=DT[dt], device="cuda")
        abi.sparoa_paged_attention(d, abi.attention_opts(64 ** -0.5), b.q.cuda(), b.k.cuda(),
                                   b.v.cuda(), b.ints(starts), b.ints(lens), table, None, None,
                                   None, out, ws)
        torch.cuda.synchronize()
        assert (out[gone[0]:min(gone[1], 15)] == 7.0).all()
        keep = [t for t in range(9) if not gone[0] <= t < gone[1]]
        check(out[keep], ref[keep], err[keep], starts)


@pytest.mark.parametrize("requests", [63, 64, 65, 200, 1500])
def test_many_requests(requests):
    g = torch.Generator().manual_seed(requests)
    rows = torch.randint(0, 3, (requests,), generator=g).tolist()
    rows[0] = 1
    keys = [n + int(e) for n, e in zip(rows, torch.randint(0, 150, (requests,), generator=g))]
    compare(Batch(rows, keys, 2, 1, 64, 16, "bf16", seed=13))


def test_equal_bits_and_split_ranges():
    """The same bits on every call and whatever the workspace held; a long cache, cut into
    ranges, equals 64 bits."""
    b = Batch([2, 1], [9000, 4000], 8, 2, 128, 16, "bf16", seed=14)
    a = compare(b)
    assert torch.equal(a, run(b, ws_fill=0)) and torch.equal(a, run(b, ws_fill=77))
    c = Batch([300], [5000], 8, 1, 64, 16, "f16", seed=15)
    a = compare(c)
    assert torch.equal(a, run(c, ws_fill=3))


def test_descriptor_bounds_do_not_change_rows():
    """Wider bounds than the batch needs: other ranges at most."""
    b = Batch([3, 20], [700, 90], 4, 2, 64, 16, "f32", seed=16, table_pages=300, spare=40)
    compare(b, max_queries=63, max_keys=4800)
    compare(b, max_queries=20, max_keys=700)


def test_other_stream_and_graph():
    abi = _abi()
    b = Batch([5, 1], [600, 2000], 8, 2, 128, 16, "bf16", seed=17)
    d = b.desc(abi)
    o = abi.attention_opts(128 ** -0.5)
    q, k, v = b.q.cuda(), b.k.cuda(), b.v.cuda()
    starts, lens, table = b.gpu()
    out = torch.zeros(6, 8, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(abi.sparoa_attention_workspace_size(d), dtype=torch.uint8, device="cuda")

    def call():
        abi.sparoa_paged_attention(d, o, q, k, v, starts, lens, table, None, None, None, out, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.synchronize()
    assert torch.equal(out, run(b))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i, (lengths, rows) in enumerate([([600, 2000], 5), ([599, 1], 5), ([6, 1999], 4),
                                         ([64, 64], 5)]):
        lens.copy_(b.ints(lengths))
        starts.copy_(b.ints([0, rows, rows + 1]))
        q.normal_()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(replayed, out) and out[:rows + 1].any(), i

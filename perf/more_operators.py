"""Timed cases of the attention side of a transformer block that serves
requests: keys and values appended to a paged cache with the rotation by
position on the way, attention over that cache, attention of drafted token
trees over it, and the move of the accepted drafts' keys and values into place.

Every case is a dict of plain values.  `prepare` makes what a program holds
before the call, `run` is one pass through an operator (through the plain
forms below, or through the public calls where `own` is set), `work` the bytes
and operations the pass cannot do without, `exact` the same outputs in 64 bits.

Kinds:
  append   q, k, v rows of many requests -> rotated q; rotated k and v in the
           pages of each request's cache
  attend   rows of many requests over their cached keys: causal or not, window,
           prefix, packed documents, capped scores, bias by distance
  tree     the drafted tokens of every request, a tree, over its cached context
           and their own ancestors
  keep     accepted drafts' keys and values move to the positions behind the
           context, in every layer

A request has `ctx` cached keys and brings between q_lo and q_hi rows; both
follow from the case alone, the values and the pages' order from the seed.
Scores spread as in a trained model (a few keys of a row count most).
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------- cases

def _append(**kw):
    return dict(dict(kind="append", rot=kw["dim"], interleaved=False, fused=True, spare=0), **kw)


def _attend(**kw):
    return dict(dict(kind="attend", causal=True, window=0, prefix=0, doc=0, cap=0.0, slopes=False,
                     spare=0), **kw)


def listed():
    return [
        # one token being generated, one request: all latency
        _append(name="append_token", requests=1, q_lo=1, q_hi=1, ctx_lo=1000, ctx_hi=1000,
                heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # a prefill of 16 requests of different lengths, a stream of rows
        _append(name="append_prefill", requests=16, q_lo=100, q_hi=900, ctx_lo=0, ctx_hi=0,
                heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # an odd fp32 batch with padding behind it: pairs side by side, part of the head
        # rotated, pages of an odd size
        _append(name="append_ragged", requests=7, q_lo=1, q_hi=131, ctx_lo=0, ctx_hi=500, heads=12,
                kv_heads=3, dim=80, page=25, dtype="f32", rot=32, interleaved=True, fused=False,
                spare=9),
        # one token over a chat's cache: latency and one request's keys over the whole card
        _attend(name="attend_token", requests=1, q_lo=1, q_hi=1, ctx_lo=4133, ctx_hi=4133,
                heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # 64 requests decoding, caches of very different lengths: a stream of keys
        _attend(name="attend_decode", requests=64, q_lo=1, q_hi=1, ctx_lo=200, ctx_hi=8000,
                heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # a prefill of two long prompts, the largest call: matrix products
        _attend(name="attend_prefill", requests=2, q_lo=4096, q_hi=4096, ctx_lo=0, ctx_hi=0,
                heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # chunks of prompts beside decoding requests: capped scores, a window, padding behind
        _attend(name="attend_chunks", requests=12, q_lo=1, q_hi=700, ctx_lo=0, ctx_hi=3000,
                heads=16, kv_heads=4, dim=64, page=32, dtype="f16", window=1024, cap=30.0,
                spare=13),
        # odd fp32 rows: bias by distance, packed documents, a prefix seen both ways
        _attend(name="attend_f32", requests=5, q_lo=30, q_hi=333, ctx_lo=0, ctx_hi=400, heads=6,
                kv_heads=6, dim=80, page=25, dtype="f32", prefix=70, doc=101, slopes=True),
        # one request's tree of 26 drafts: latency
        dict(name="tree_one", kind="tree", requests=1, q_lo=26, q_hi=26, ctx_lo=2000, ctx_hi=2000,
             heads=32, kv_heads=8, dim=128, page=16, dtype="bf16", cap=0.0, window=0, slopes=False,
             spare=0),
        # 32 requests with trees of up to 60 drafts
        dict(name="tree_batch", kind="tree", requests=32, q_lo=40, q_hi=60, ctx_lo=200,
             ctx_hi=5000, heads=32, kv_heads=8, dim=128, page=16, dtype="bf16", cap=0.0, window=0,
             slopes=False, spare=0),
        # the accepted path of one request, one layer: all latency
        dict(name="keep_one", kind="keep", requests=1, q_lo=26, q_hi=26, ctx_lo=100, ctx_hi=100,
             kv_heads=8, dim=128, page=16, dtype="bf16", layers=1, accepted=4),
        # 64 requests, 16 layers in one call
        dict(name="keep_batch", kind="keep", requests=64, q_lo=40, q_hi=60, ctx_lo=10, ctx_hi=90,
             kv_heads=8, dim=128, page=16, dtype="bf16", layers=16, accepted=6),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _heads(rng):
    """(heads, kv_heads, dim)"""
    kv = rng.choice((1, 2, 3, 4, 8, 8))
    group = rng.choice((1, 2, 4, 4, 5, 8))
    dim = rng.choice((64, 64, 128, 128, 128, 80, 96, 40, 192, 256))
    return kv * group, kv, dim


def draw(rng):
    kind = rng.choice(("append", "append", "attend", "attend", "attend", "tree", "tree", "keep"))
    dt = rng.choice(("bf16", "bf16", "f16", "f16", "f32"))
    heads, kv, dim = _heads(rng)
    page = rng.choice((16, 16, 32, 64, 25, 1, 256))
    spare = rng.choice((0, 0, 0, 11))
    if kind == "append":
        requests = _log(rng, 1, 64)
        rows = _log(rng, 1, max(1, 8000 // requests))
        return dict(kind="append", requests=requests, q_lo=max(1, rows // 2), q_hi=rows, ctx_lo=0,
                    ctx_hi=rng.choice((0, 300, 1500)), heads=heads, kv_heads=kv, dim=dim,
                    page=page, dtype=dt, rot=rng.choice((dim, dim, dim // 2, 0)),
                    interleaved=rng.random() < 0.4, fused=rng.random() < 0.6, spare=spare)
    if kind == "attend":
        shape = rng.choice(("decode", "decode", "prefill", "chunks"))
        if shape == "decode":
            requests = _log(rng, 1, 96)
            ctx = _log(rng, 16, max(32, int(3e8 / (requests * kv * dim * _SIZE[dt]))))
            ctx = min(ctx, 65536)
            q_lo, q_hi = 1, rng.choice((1, 1, 1, 3))
        elif shape == "prefill":
            requests, ctx = _log(rng, 1, 16), 0
            # rows^2 heads dim requests below the largest listed case's, fp32 a tenth
            most = (2.0 * 4096 * 4096 * 32 * 128) * (0.1 if dt == "f32" else 1.0)
            q_hi = _log(rng, 64, max(65, min(8192, int((most / (requests * heads * dim)) ** 0.5))))
            q_lo = max(1, q_hi // 3)
        else:
            requests, ctx = _log(rng, 1, 24), _log(rng, 64, 4000)
            most = (0.5 * 4096 * 4096 * 32 * 128) * (0.1 if dt == "f32" else 1.0)
            q_lo, q_hi = 1, _log(rng, 16, max(17, min(2048, int(most / (requests * heads * dim *
                                                                        (ctx + 1000))))))
        return _attend(requests=requests, q_lo=q_lo, q_hi=q_hi, ctx_lo=ctx // 8, ctx_hi=ctx,
                       heads=heads, kv_heads=kv, dim=dim, page=page, dtype=dt,
                       causal=rng.random() < 0.85, window=rng.choice((0, 0, 0, 100, 1024)),
                       prefix=rng.choice((0, 0, 0, 50)), doc=rng.choice((0, 0, 0, 300)),
                       cap=rng.choice((0.0, 0.0, 20.0, 50.0)), slopes=rng.random() < 0.25,
                       spare=spare)
    if kind == "tree":
        requests = _log(rng, 1, 48)
        nodes = rng.choice((8, 26, 60, 64, 100))
        ctx = _log(rng, 32, max(64, int(2e8 / (requests * kv * dim * _SIZE[dt] *
                                               (4 if dt == "f32" else 1)))))
        ctx = min(ctx, 32768, int(6e11 / (requests * nodes * heads * dim * 4)))
        return dict(kind="tree", requests=requests, q_lo=max(1, nodes // 2), q_hi=nodes,
                    ctx_lo=ctx // 8, ctx_hi=ctx, heads=heads, kv_heads=kv, dim=dim, page=page,
                    dtype=dt, cap=rng.choice((0.0, 0.0, 30.0)), window=rng.choice((0, 0, 500)),
                    slopes=rng.random() < 0.25, spare=spare)
    nodes = rng.choice((8, 26, 60, 64, 100))
    requests = _log(rng, 1, 64)
    page = max(page, 16)
    ctx = rng.choice((0, 40, 200))
    most = int(2.5e8 / (requests * (ctx + nodes + page) * kv * dim * _SIZE[dt]))
    return dict(kind="keep", requests=requests, q_lo=nodes, q_hi=nodes, ctx_lo=ctx // 2, ctx_hi=ctx,
                kv_heads=kv, dim=dim, page=page, dtype=dt, layers=_log(rng, 1, max(1, min(24, most))),
                accepted=rng.randint(1, max(1, min(8, nodes // 2))))


# ---------------------------------------------------------------- geometry

def _spread(lo, hi, r, n, step):
    """Request r's share of [lo, hi]: hi for the first, the others spread."""
    return hi if r == 0 else lo + int((hi - lo) * math.fmod(r * step, 1.0))


def _lengths(case):
    """(rows, context) of every request."""
    n = case["requests"]
    rows = [_spread(case["q_lo"], case["q_hi"], r, n, 0.7548776662) for r in range(n)]
    ctx = [_spread(case["ctx_lo"], case["ctx_hi"], r, n, 0.6180339887) for r in range(n)]
    return rows, ctx


def _parents(nodes, r):
    """A tree in order of depth: 2 to 4 drafts behind each, by request."""
    return [(i - 1) // (2 + r % 3) for i in range(nodes)]


def _depths(nodes, r):
    d = []
    for i, p in enumerate(_parents(nodes, r)):
        d.append(0 if i == 0 else d[p] + 1)
    return d


def _accepted(case, rows):
    """Accepted drafts of every request: j itself, or one past the accepted ones (so that a
    second pass finds the same)."""
    out = []
    for r, n in enumerate(rows):
        a = min(case["accepted"] - (r % 2 if case["accepted"] > 1 else 0), max(1, n // 2))
        out.append([0] + [a + (j * 7 + r) % (n - a) for j in range(1, a)] if n > a else [0])
        out[-1][1:] = sorted(set(out[-1][1:]))
        for j in range(1, len(out[-1])):
            out[-1][j] = max(out[-1][j], len(out[-1]))
    return out


def _interval(case, ctx, n, j):
    """[lo, hi) of the keys that row j of a request sees."""
    length, p = ctx + n, ctx + j
    hi = min(length, max(p + 1, case["prefix"])) if case["causal"] else length
    lo = max(0, p + 1 - case["window"]) if case["window"] else 0
    return max(lo, p - p % case["doc"]) if case["doc"] else lo, hi


# ------------------------------------------------------------------ inputs

def _inputs(case, seed):
    """The case's tensors on the GPU: values and pages from the seed, shapes from the case."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(0x5EED1000 + seed)
    dt = _DT[case["dtype"]]
    rows, ctx = _lengths(case)
    keys = [a + b for a, b in zip(rows, ctx)]
    kv, dim, page = case["kv_heads"], case["dim"], case["page"]

    def normal(*shape, std=1.0, to=dt):
        return torch.empty(shape, dtype=to, device=dev).normal_(0.0, std, generator=g)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    # every request's pages, from anywhere in the cache; a few pages are nobody's
    per = [-(-k // page) for k in keys]
    pages = sum(per) + 3
    order = torch.randperm(pages, device=dev, generator=g).to(torch.int32)
    table = torch.zeros(len(keys), max(per), dtype=torch.int32, device=dev)
    at = 0
    for r, p in enumerate(per):
        table[r, :p] = order[at:at + p]
        at += p
    start = [0]
    for n in rows:
        start.append(start[-1] + n)
    s = dict(rows=rows, ctx=ctx, keys=keys, pages=pages, table=table, q_start=ints(start),
             kv_len=ints(keys))
    layers = (case["layers"],) if case["kind"] == "keep" else ()
    s["k_cache"] = normal(*layers, pages, kv, page, dim)
    s["v_cache"] = normal(*layers, pages, kv, page, dim)
    if case["kind"] == "keep":
        accepted = _accepted(case, rows)
        most = max(len(a) for a in accepted)
        s["keep"] = ints([a + [-1] * (most - len(a)) for a in accepted])
        s["kept"] = ints([len(a) for a in accepted])
        s["accepted"] = accepted
        return s
    heads = case["heads"]
    tokens = start[-1] + case["spare"]
    s["tokens"] = tokens
    if case["kind"] == "append":
        if case["fused"]:      # the rows of one projection
            qkv = normal(tokens, (heads + 2 * kv) * dim)
            s["q"], s["k"], s["v"] = qkv.split([heads * dim, kv * dim, kv * dim], 1)
        else:
            s["q"], s["k"], s["v"] = (normal(tokens, h * dim) for h in (heads, kv, kv))
        half = case["rot"] // 2
        s["freqs"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=dev) / max(1, half))
        s["q_out"] = torch.zeros(tokens, heads, dim, dtype=dt, device=dev)
        return s
    s["q"] = normal(tokens, heads, dim, std=2.0)
    s["out"] = torch.zeros(tokens, heads, dim, dtype=dt, device=dev)
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, heads + 1, device=dev) / heads)).float() \
        if case["slopes"] else None
    if case["kind"] == "tree":
        words = -(-max(rows) // 64)
        mask, pos = torch.zeros(tokens, words, dtype=torch.int64), torch.zeros(tokens,
                                                                               dtype=torch.int32)
        for r, n in enumerate(rows):
            sees = []
            for i, p in enumerate(_parents(n, r)):
                sees.append((0 if i == 0 else sees[p]) | 1 << i)
                for w in range(words):
                    v = sees[i] >> (64 * w) & (1 << 64) - 1
                    mask[start[r] + i, w] = v - (1 << 64) if v >> 63 else v
            pos[start[r]:start[r] + n] = ctx[r] + torch.tensor(_depths(n, r), dtype=torch.int32)
        s["mask"], s["pos"] = mask.to(dev), pos.to(dev)
        return s
    s["prefix"] = ints([case["prefix"]] * len(rows)) if case["prefix"] else None
    s["first"] = None
    if case["doc"]:
        p = torch.cat([torch.arange(c, c + n) for c, n in zip(ctx, rows)] +
                      [torch.zeros(case["spare"], dtype=torch.int64)])
        s["first"] = (p - p % case["doc"]).to(torch.int32).to(dev)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    from paper_2511_19457_amd import abi
    s["abi"] = abi
    s["desc"] = abi.kv_desc(s.get("tokens", sum(s["rows"])), case["requests"],
                            case.get("heads", case["kv_heads"]), case["kv_heads"], case["dim"],
                            s["pages"], case["page"], s["table"].shape[1], _DT[case["dtype"]],
                            max_queries=max(s["rows"]), max_keys=max(s["keys"]))
    if case["kind"] in ("attend", "tree"):
        s["opts"] = abi.attention_opts(scale=case["dim"] ** -0.5, cap=case["cap"],
                                       window=case["window"], causal=case.get("causal", True))
        s["ws"] = torch.empty(max(16, abi.sparoa_attention_workspace_size(s["desc"])),
                              dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------- passes

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


def _own_append(s):
    c = s["case"]
    s["abi"].sparoa_kv_append(s["desc"], s["q"], s["k"], s["v"], s["freqs"] if c["rot"] else None,
                              None, s["q_start"], s["kv_len"], s["table"], s["q_out"],
                              s["k_cache"], s["v_cache"], rot_dim=c["rot"],
                              interleaved=c["interleaved"])
    return s["q_out"], s["k_cache"], s["v_cache"]


def _own_attend(s):
    s["abi"].sparoa_paged_attention(s["desc"], s["opts"], s["q"], s["k_cache"], s["v_cache"],
                                    s["q_start"], s["kv_len"], s["table"], s["prefix"], s["first"],
                                    s["slopes"], s["out"], s["ws"])
    return s["out"]


def _own_tree(s):
    s["abi"].sparoa_tree_attention(s["desc"], s["opts"], s["q"], s["k_cache"], s["v_cache"],
                                   s["q_start"], s["kv_len"], s["table"], s["mask"], s["pos"],
                                   s["slopes"], s["out"], s["ws"])
    return s["out"]


def _own_keep(s):
    s["abi"].sparoa_kv_keep(s["desc"], s["case"]["layers"], s["q_start"], s["kv_len"], s["table"],
                            s["keep"], s["kept"], s["k_cache"], s["v_cache"])
    return s["k_cache"], s["v_cache"]


_OWN = dict(append=_own_append, attend=_own_attend, tree=_own_tree, keep=_own_keep)


def _rotated(x, angles, rot, interleaved):
    """x [tokens, heads, dim] fp32, angles [tokens, rot / 2] fp64"""
    if not rot:
        return x
    c, s = torch.cos(angles).float()[:, None], torch.sin(angles).float()[:, None]
    if interleaved:
        a, b = x[:, :, 0:rot:2], x[:, :, 1:rot:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], 3).reshape(*x.shape[:2], rot)
    else:
        a, b = x[:, :, :rot // 2], x[:, :, rot // 2:rot]
        turned = torch.cat([a * c - b * s, a * s + b * c], 2)
    return torch.cat([turned, x[:, :, rot:]], 2)


def _new_rows(s):
    """(request, position) of every row of the requests."""
    req = torch.repeat_interleave(torch.arange(len(s["rows"]), device="cuda"),
                                  s["q_start"][1:] - s["q_start"][:-1],
                                  output_size=sum(s["rows"]))
    back = (s["kv_len"] - s["q_start"][1:])[req]
    return req, torch.arange(req.numel(), device="cuda") + back


def _plain_append(s):
    c = s["case"]
    req, pos = _new_rows(s)
    n, page = req.numel(), c["page"]
    angles = pos.double()[:, None] * s["freqs"]
    q, k, v = (s[t][:n].reshape(n, -1, c["dim"]) for t in ("q", "k", "v"))
    s["q_out"][:n] = _rotated(q.float(), angles, c["rot"], c["interleaved"]).to(q.dtype)
    to, off = s["table"][req, pos // page].long(), pos % page
    s["k_cache"][to, :, off] = _rotated(k.float(), angles, c["rot"], c["interleaved"]).to(k.dtype)
    s["v_cache"][to, :, off] = v
    return s["q_out"], s["k_cache"], s["v_cache"]


def _groups(s, c):
    """Requests side by side, padded to the longest, while they fit 1.5e9 numbers."""
    out, n, length = [], 0, 0
    for r, (a, b) in enumerate(zip(s["rows"], s["keys"])):
        n2, l2 = max(n, a), max(length, b)
        size = (len(out[-1]) + 1 if out else 1) * l2 * (n2 * c["heads"] + 2 * c["kv_heads"] * c["dim"])
        if out and size <= 1.5e9:
            out[-1].append(r)
            n, length = n2, l2
        else:
            out.append([r])
            n, length = a, b
    return out


def _plain_scores(s, reqs):
    """One padded group: rows [b, n], their positions, keys' positions, scores and values."""
    c, dev = s["case"], s["q"].device
    kv, dim, page = c["kv_heads"], c["dim"], c["page"]
    n, length = max(s["rows"][r] for r in reqs), max(s["keys"][r] for r in reqs)
    rows, lens = s["q_start"][reqs[0]:reqs[-1] + 2].long(), s["kv_len"][reqs[0]:reqs[-1] + 1].long()
    j, k = torch.arange(n, device=dev), torch.arange(length, device=dev)
    live = j < (rows[1:] - rows[:-1])[:, None]
    row = torch.where(live, rows[:-1, None] + j, 0)
    inside = k < lens[:, None]
    at = torch.where(inside, k, 0)
    to = s["table"][reqs[0]:reqs[-1] + 1].long().gather(1, at // page)
    keys = s["k_cache"][to, :, at % page].float().permute(0, 2, 3, 1).contiguous()
    values = s["v_cache"][to, :, at % page].float().permute(0, 2, 1, 3).contiguous()
    values = torch.where(inside[:, None, :, None], values, 0.0)
    q = s["q"][row].float().reshape(len(reqs), n, kv, -1, dim).permute(0, 2, 3, 1, 4)
    group = q.shape[2]
    x = torch.matmul(q.reshape(len(reqs), kv, group * n, dim), keys) * dim ** -0.5
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    base = lens - (rows[1:] - rows[:-1])
    return live, row, base, j, k, inside, x.reshape(len(reqs), kv * group, n, length), values


def _plain_join(s, live, row, x, values):
    """softmax and its product with the values, to the rows of out"""
    b, heads, n, length = x.shape
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(top > float("-inf"), top, 0.0))
    total = p.sum(3, keepdim=True)
    y = torch.matmul(p.reshape(b, values.shape[1], -1, length), values).reshape(b, heads, n, -1)
    y = torch.where(total > 0, y / total, 0.0).permute(0, 2, 1, 3).to(s["out"].dtype)
    s["out"][row[live]] = y[live]


def _plain_attend(s):
    c = s["case"]
    for reqs in _groups(s, c):
        live, row, base, j, k, inside, x, values = _plain_scores(s, reqs)
        p = base[:, None] + j
        sees = inside[:, None].expand(-1, j.numel(), -1)
        if c["causal"]:
            ahead = k <= p[:, :, None]
            sees = sees & (ahead | (k < c["prefix"]) if c["prefix"] else ahead)
        if c["window"]:
            sees = sees & (k > (p - c["window"])[:, :, None])
        if c["doc"]:
            sees = sees & (k >= s["first"][row][:, :, None])
        if c["slopes"]:
            x = x - s["slopes"][:, None, None] * (p[:, :, None] - k).abs()[:, None].float()
        _plain_join(s, live, row, torch.where(sees[:, None], x, float("-inf")), values)
    return s["out"]


def _plain_tree(s):
    c = s["case"]
    for reqs in _groups(s, c):
        live, row, base, j, k, inside, x, values = _plain_scores(s, reqs)
        node = (k - base[:, None]).clamp(min=0)                          # [b, keys]
        most = s["mask"].shape[1] * 64 - 1
        node = node.clamp(max=most)[:, None].expand(-1, j.numel(), -1)
        bits = s["mask"][row].gather(2, node // 64) >> (node % 64) & 1
        p = s["pos"][row].long()
        start = row[:, :1]
        of_key = s["pos"][(start + node[:, 0]).clamp(max=s["pos"].numel() - 1)].long()
        of_key = torch.where(k < base[:, None], k, of_key)               # a key's position
        sees = inside[:, None] & ((k < base[:, None])[:, None] | (bits != 0))
        if c["window"]:
            sees = sees & (of_key[:, None] > (p - c["window"])[:, :, None])
        if c["slopes"]:
            far = (p[:, :, None] - of_key[:, None]).abs().float()
            x = x - s["slopes"][:, None, None] * far[:, None]
        _plain_join(s, live, row, torch.where(sees[:, None], x, float("-inf")), values)
    return s["out"]


def _plain_keep(s):
    page = s["case"]["page"]
    most = s["keep"].shape[1]
    base = (s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1]))[:, None].long()
    j = torch.arange(most, device="cuda")
    there = j < s["kept"][:, None]
    src = torch.where(there, base + s["keep"], base)
    dst = torch.where(there, base + j, base)        # (the first draft stays where it is)
    table = s["table"].long()
    a, b = table.gather(1, src // page), table.gather(1, dst // page)
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, b, :, dst % page] = cache[:, a, :, src % page]
    return s["k_cache"], s["v_cache"]


_PLAIN = dict(append=_plain_append, attend=_plain_attend, tree=_plain_tree, keep=_plain_keep)


# --------------------------------------------------------------- work, exact

def work(case):
    size = _SIZE[case["dtype"]]
    rows, ctx = _lengths(case)
    kv, dim = case["kv_heads"], case["dim"]
    if case["kind"] == "keep":
        moved = sum(len(a) - 1 for a in _accepted(case, rows))
        return dict(bytes=4 * moved * case["layers"] * kv * dim * size + 4 * sum(rows), flops=0)
    heads = case["heads"]
    if case["kind"] == "append":
        return dict(bytes=2 * sum(rows) * (heads + 2 * kv) * dim * size + 8 * sum(rows),
                    flops=3 * sum(rows) * (heads + kv) * case["rot"])
    pairs = keys = 0
    for r, (n, c) in enumerate(zip(rows, ctx)):
        if case["kind"] == "tree":
            pairs += n * c + sum(d + 1 for d in _depths(n, r))
            keys += c + n
        else:
            spans = [_interval(case, c, n, j) for j in range(n)]
            pairs += sum(max(0, b - a) for a, b in spans)
            keys += max(b for _, b in spans) - min(a for a, _ in spans)
    return dict(bytes=2 * (keys * kv + sum(rows) * heads) * dim * size,
                flops=4 * pairs * heads * dim)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "keep":
        return None
    rows, ctx, page, dim = s["rows"], s["ctx"], case["page"], case["dim"]
    starts = s["q_start"].tolist()
    if case["kind"] == "append":
        q_out, kc, vc = (s[t].double() for t in ("q_out", "k_cache", "v_cache"))
        for r, n in enumerate(rows):
            pos = torch.arange(ctx[r], ctx[r] + n, device="cuda")
            mine = slice(starts[r], starts[r] + n)
            turn = torch.polar(torch.ones(n, case["rot"] // 2, dtype=torch.float64, device="cuda"),
                               torch.outer(pos.double(), s["freqs"]))[:, None]

            def spun(x):
                x = x.double().reshape(n, -1, dim).clone()
                h = case["rot"] // 2
                a, b = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if case["interleaved"] else \
                    (slice(0, h), slice(h, 2 * h))
                z = torch.complex(x[:, :, a].contiguous(), x[:, :, b].contiguous()) * turn
                x[:, :, a], x[:, :, b] = z.real, z.imag
                return x

            q_out[mine] = spun(s["q"][mine])
            to = s["table"][r].long()[pos // page]
            kc[to, :, pos % page] = spun(s["k"][mine])
            vc[to, :, pos % page] = s["v"][mine].double().reshape(n, -1, dim)
        return q_out, kc, vc
    out = s["out"].double()
    group = case["heads"] // case["kv_heads"]
    low = float("-inf")
    for r, n in enumerate(rows):
        length = ctx[r] + n
        k = torch.arange(length, device="cuda")
        to = s["table"][r].long()[k // page]
        if case["kind"] == "tree":
            sees = torch.ones(n, length, dtype=torch.bool)
            own_pos = torch.tensor([ctx[r] + d for d in _depths(n, r)])
            sees[:, ctx[r]:] = False
            for i, p in enumerate(_parents(n, r)):
                if i:
                    sees[i, ctx[r]:] = sees[p, ctx[r]:]
                sees[i, ctx[r] + i] = True
            key_pos = torch.cat([torch.arange(ctx[r]), own_pos])
            far = (own_pos[:, None] - key_pos).cuda()
            sees = sees.cuda()
            if case["window"]:
                sees &= far < case["window"]
        else:
            spans = torch.tensor([_interval(case, ctx[r], n, j) for j in range(n)], device="cuda")
            sees = (k >= spans[:, :1]) & (k < spans[:, 1:])
            far = torch.arange(ctx[r], length, device="cuda")[:, None] - k
        mine = slice(starts[r], starts[r] + n)
        for h in range(case["heads"]):
            keys = s["k_cache"][to, h // group, k % page].double()
            x = s["q"][mine, h].double() @ keys.t() / math.sqrt(dim)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if case["slopes"]:
                x = x - float(s["slopes"][h]) * far.abs()
            w = torch.softmax(torch.where(sees, x, low), 1)
            w = torch.where(sees.any(1, keepdim=True), w, torch.zeros_like(w))
            out[mine, h] = w @ s["v_cache"][to, h // group, k % page].double()
    return out

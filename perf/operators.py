"""Timed cases of the transformer-block operators: routing to experts and its
dispatch plan, the experts' products, FCs with low-rank adapters of many
requests, and the norm between two blocks.

Every case is a dict of plain values.  `prepare` makes what a program holds
before the call, `run` is one pass through an operator (through the plain
forms below, or through the public calls where `own` is set), `work` the bytes
and operations the pass cannot do without, `exact` the same outputs in 64 bits.

Kinds:
  route    logits of T tokens over E experts -> chosen experts, their weights,
           and the plan that sorts the (token, choice) slots by expert
  experts  chosen experts and weights of T tokens -> plan, gated or plain FFN
           of each token's experts, weighted sum (plus residual)
  adapter  y = act(x W^T + bias + scale_a (x A_a^T) B_a^T + residual), the
           adapter a of each row its own (or none)
  norm     r' = c r + gate * post_norm(y), n = pre_norm(r')

Inputs are seeded: unit normals as activations, He-scaled weights, logits of
a trained router's spread, requests as runs of rows in a prefill batch and as
single rows in a decode batch.
"""
import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ------------------------------------------------------------------- cases

def listed():
    return [
        # the router of one token being generated: all latency
        dict(name="route_token", kind="route", tokens=1, experts=64, top_k=8, score="softmax",
             groups=1, top_groups=1, group_best=1, bias=False, renorm=True, scale=1.0, pad=0.0,
             off=0, dtype="bf16"),
        # an odd batch whose tail is padding, odd expert count, two experts switched off
        dict(name="route_ragged", kind="route", tokens=1003, experts=60, top_k=4, score="softmax",
             groups=1, top_groups=1, group_best=1, bias=False, renorm=False, scale=1.0, pad=0.2,
             off=2, dtype="f16"),
        # a long prefill over many experts: sigmoid scores, balance bias, 4 of 8 groups
        dict(name="route_groups", kind="route", tokens=16384, experts=256, top_k=8,
             score="sigmoid", groups=8, top_groups=4, group_best=2, bias=True, renorm=True,
             scale=2.5, pad=0.0, off=0, dtype="f32"),
        # one token through its 8 of 64 experts: a stream of weights
        dict(name="experts_token", kind="experts", tokens=1, experts=64, top_k=8, hidden=2048,
             inner=1024, gated=True, act="silu", bias=False, residual=True, pad=0.0, dtype="bf16"),
        # 64 requests decoding: every expert's weights for a few rows each
        dict(name="experts_decode", kind="experts", tokens=64, experts=64, top_k=8, hidden=2048,
             inner=1024, gated=True, act="silu", bias=False, residual=True, pad=0.0, dtype="bf16"),
        # a prefill of 4096 tokens, the largest call: matrix products
        dict(name="experts_prefill", kind="experts", tokens=4096, experts=64, top_k=8,
             hidden=2048, inner=1024, gated=True, act="silu", bias=False, residual=True, pad=0.0,
             dtype="bf16"),
        # an odd, padded batch through ungated experts with biases, the FFN stack's width
        dict(name="experts_ragged", kind="experts", tokens=777, experts=20, top_k=2, hidden=768,
             inner=1000, gated=False, act="gelu", bias=True, residual=False, pad=0.15,
             dtype="f16"),
        # 32 requests decoding, 24 adapters over one projection, some rows with none
        dict(name="adapter_decode", kind="adapter", m=32, k=4096, n=4096, adapters=24, rank=16,
             requests=32, bare=0.2, act="none", bias=False, residual=True, dtype="bf16"),
        # a prefill of 16 requests of different lengths, each with its adapter
        dict(name="adapter_prefill", kind="adapter", m=4096, k=4096, n=4096, adapters=16, rank=32,
             requests=16, bare=0.1, act="none", bias=False, residual=False, dtype="bf16"),
        # an odd fp32 batch with bias and ReLU
        dict(name="adapter_f32", kind="adapter", m=333, k=768, n=1000, adapters=5, rank=8,
             requests=9, bare=0.2, act="relu", bias=True, residual=False, dtype="f32"),
        # the norm between two blocks of one token: all latency
        dict(name="norm_token", kind="norm", rows=1, cols=2048, post="rms", pre="rms", gate=True,
             gate_rows=1, c=1.0, dtype="bf16"),
        # the same of a long prefill: a stream of activations
        dict(name="norm_prefill", kind="norm", rows=8192, cols=4096, post="rms", pre="rms",
             gate=True, gate_rows=8192, c=1.0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _width(rng, lo, hi):
    """A feature width of [lo, hi]: a multiple of 8, one in eight of them any integer."""
    return _log(rng, lo, hi) if rng.random() < 0.125 else 8 * _log(rng, -(-lo // 8), hi // 8)


def draw(rng):
    kind = rng.choice(("route", "experts", "experts", "adapter", "adapter", "norm"))
    dt = rng.choice(("bf16", "bf16", "f16", "f16", "f32"))
    if kind == "route":
        groups = rng.choice((1, 1, 1, 2, 4, 8))
        experts = groups * _log(rng, max(2, 8 // groups), 512 // groups)
        top_groups = rng.randint(1, groups)
        score = rng.choice(("softmax", "sigmoid"))
        best = rng.choice((1, 2)) if score == "sigmoid" and groups > 1 else 1
        return dict(kind="route", tokens=_log(rng, 1, 16384), experts=experts,
                    top_k=rng.randint(1, min(12, experts // groups * top_groups)), score=score,
                    groups=groups, top_groups=top_groups, group_best=best,
                    bias=score == "sigmoid" and rng.random() < 0.5, renorm=rng.random() < 0.7,
                    scale=rng.choice((1.0, 2.5)), pad=rng.choice((0.0, 0.0, 0.25)),
                    off=rng.choice((0, 0, 1)), dtype=dt)
    if kind == "experts":
        experts = _log(rng, 4, 128)
        top_k = rng.randint(1, min(8, experts))
        gated = rng.random() < 0.6
        cap = 1.0e10 if dt == "f32" else 2.0e11
        hidden, inner = _width(rng, 256, 2560), _width(rng, 200, 2048)
        while experts * hidden * inner * (3 if gated else 2) > (1.7e8 if dt == "f32" else 3.5e8):
            experts = max(4, experts // 2)
            top_k = min(top_k, experts)
        per = 2.0 * top_k * hidden * inner * (3 if gated else 2)
        if hidden % 8 or inner % 8:
            cap /= 16
        return dict(kind="experts", tokens=_log(rng, 1, max(2, min(6000, int(cap / per)))),
                    experts=experts, top_k=top_k, hidden=hidden, inner=inner, gated=gated,
                    act="silu" if gated else rng.choice(("relu", "gelu")),
                    bias=rng.random() < 0.3, residual=rng.random() < 0.5,
                    pad=rng.choice((0.0, 0.0, 0.2)), dtype=dt)
    if kind == "adapter":
        k, n = _width(rng, 256, 6144), _width(rng, 128, 6144)
        cap = 1.0e10 if dt == "f32" else 1.2e11
        if k % 8 or n % 8:
            cap /= 16
        m = _log(rng, 1, max(2, min(8192, int(cap / (2.0 * k * n)))))
        adapters = _log(rng, 1, 64)
        return dict(kind="adapter", m=m, k=k, n=n, adapters=adapters,
                    rank=rng.choice((4, 8, 16, 16, 32, 64)),
                    requests=m if m <= 64 else _log(rng, 1, 64), bare=rng.choice((0.0, 0.2, 0.5)),
                    act=rng.choice(("none", "none", "relu")), bias=rng.random() < 0.3,
                    residual=rng.random() < 0.4, dtype=dt)
    cols = _width(rng, 64, 8192)
    rows = _log(rng, 1, max(2, min(16384, (32 << 20) // cols)))
    gate_rows = rng.choice((rows, 1, max(1, rows // 4)))
    return dict(kind="norm", rows=rows, cols=cols, post=rng.choice(("none", "rms", "layer")),
                pre=rng.choice(("rms", "layer")), gate=rng.random() < 0.6, gate_rows=gate_rows,
                c=rng.choice((1.0, 0.5)), dtype=dt)


# ------------------------------------------------------------------ inputs

def _inputs(case, seed):
    """The case's tensors on the GPU, from the seed alone."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(0x5EED0000 + seed)
    dt = _DT[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, to=dt):
        t = torch.empty(shape, dtype=to, device=dev)
        return t.normal_(mean, std, generator=g)

    def rand(*shape):
        return torch.rand(shape, device=dev, generator=g)

    if case["kind"] == "route":
        t, e = case["tokens"], case["experts"]
        logits = normal(t, e, std=1.5)
        if case["off"]:
            logits[:, torch.randperm(e, device=dev, generator=g)[:case["off"]]] = float("-inf")
        s = dict(logits=logits,
                 bias=normal(e, std=0.1, to=torch.float32) if case["bias"] else None,
                 valid=(torch.arange(t, device=dev) < t - int(case["pad"] * t)).to(torch.uint8)
                 if case["pad"] else None)
        return s
    if case["kind"] == "experts":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        h, i = case["hidden"], case["inner"]
        up = 2 * i if case["gated"] else i
        # experts of uneven popularity, distinct for each token
        pop = normal(e, std=0.4, to=torch.float32) + normal(t, e, to=torch.float32)
        idx = torch.argsort(pop, dim=1, descending=True)[:, :k].to(torch.int32).contiguous()
        w = rand(t, k) + 0.1
        w = w / w.sum(1, keepdim=True)
        if case["pad"]:
            off = torch.arange(t, device=dev) >= t - int(case["pad"] * t)
            idx[off] = -1
            w[off] = 0
        return dict(x=normal(t, h), w_up=normal(e, up, h, std=(2.0 / h) ** 0.5),
                    w_down=normal(e, h, i, std=i ** -0.5),
                    b_up=normal(e, up, std=0.1) if case["bias"] else None,
                    b_down=normal(e, h, std=0.1) if case["bias"] else None,
                    residual=normal(t, h) if case["residual"] else None, idx=idx, weights=w)
    if case["kind"] == "adapter":
        m, k, n, na, r = case["m"], case["k"], case["n"], case["adapters"], case["rank"]
        req = case["requests"]
        ids = torch.randint(na, (req,), device=dev, generator=g, dtype=torch.int32)
        ids[rand(req) < case["bare"]] = -1
        # rows of a request are consecutive, requests of uneven length
        cut = torch.sort((rand(req) * m).to(torch.int64)).values
        of = torch.searchsorted(cut, torch.arange(m, device=dev), right=True) - 1
        of = torch.arange(m, device=dev) if req == m else of.clamp(min=0)
        return dict(x=normal(m, k), w=normal(n, k, std=k ** -0.5),
                    bias=normal(n, std=0.1) if case["bias"] else None,
                    a=normal(na, r, k, std=k ** -0.5), b=normal(na, n, r, std=0.5 * r ** -0.5),
                    scale=rand(na) + 0.5, ids=ids[of].contiguous(),
                    residual=normal(m, n) if case["residual"] else None)
    r, c = case["rows"], case["cols"]
    layer_post, layer_pre = case["post"] == "layer", case["pre"] == "layer"
    return dict(y=normal(r, c, std=2.0), r=normal(r, c),
                post_w=normal(c, std=0.1, mean=1.0) if case["post"] != "none" else None,
                post_b=normal(c, std=0.1) if layer_post else None,
                gate=normal(-(-r // case["gate_rows"]), c, std=0.3) if case["gate"] else None,
                pre_w=normal(c, std=0.1, mean=1.0),
                pre_b=normal(c, std=0.1) if layer_pre else None)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    dev = torch.device("cuda")
    dt = _DT[case["dtype"]]
    if not own:
        return s
    from paper_2511_19457_amd import abi
    s["abi"] = abi

    def scratch(size):
        return torch.empty(max(16, size), dtype=torch.uint8, device=dev)

    if case["kind"] == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        s["desc"] = abi.expert_route_desc(
            t, e, k, dt, score=abi.SCORE_SIGMOID if case["score"] == "sigmoid"
            else abi.SCORE_SOFTMAX, groups=case["groups"], top_groups=case["top_groups"],
            group_best=case["group_best"], renormalise=case["renorm"], scale=case["scale"])
        s["idx"] = torch.empty(t, k, dtype=torch.int32, device=dev)
        s["weights"] = torch.empty(t, k, dtype=torch.float32, device=dev)
        s["plan"] = torch.empty(abi.sparoa_expert_plan_words(t, k, e), dtype=torch.int32,
                                device=dev)
        s["views"] = abi.expert_plan_views(s["plan"], t, k, e)
        s["ws"] = scratch(abi.sparoa_expert_route_workspace_size(s["desc"]))
    elif case["kind"] == "experts":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        s["act"] = {"silu": abi.ACT_SILU, "gelu": abi.ACT_GELU, "relu": abi.ACT_RELU}[case["act"]]
        s["desc"] = abi.expert_ffn_desc(t, k, e, case["hidden"], case["inner"], dt,
                                        gated=case["gated"], has_bias=case["bias"])
        s["plan"] = torch.empty(abi.sparoa_expert_plan_words(t, k, e), dtype=torch.int32,
                                device=dev)
        s["plan_ws"] = scratch(abi.sparoa_expert_plan_workspace_size(t, k, e))
        s["ws"] = scratch(abi.sparoa_expert_ffn_workspace_size(s["desc"]))
        s["out"] = torch.empty(t, case["hidden"], dtype=dt, device=dev)
    elif case["kind"] == "adapter":
        s["act"] = {"none": abi.ACT_NONE, "relu": abi.ACT_RELU}[case["act"]]
        s["desc"] = abi.fc_adapted_desc(case["m"], case["k"], case["n"], case["adapters"],
                                        case["rank"], dt, has_bias=case["bias"])
        s["ws"] = scratch(abi.sparoa_fc_adapted_workspace_size(s["desc"]))
        s["out"] = torch.empty(case["m"], case["n"], dtype=dt, device=dev)
    else:
        norm = {"none": abi.NORM_NONE, "rms": abi.NORM_RMS, "layer": abi.NORM_LAYER}
        s["desc"] = abi.block_norm_desc(case["rows"], case["cols"], dt, post=norm[case["post"]],
                                        pre=norm[case["pre"]], eps=1e-6,
                                        gate_rows=case["gate_rows"], residual_scale=case["c"])
        s["r_out"], s["n_out"] = torch.empty_like(s["r"]), torch.empty_like(s["r"])
    return s


# ------------------------------------------------------------------- passes

def run(state):
    return _OWN[state["case"]["kind"]](state) if own else _PLAIN[state["case"]["kind"]](state)


def _own_route(s):
    s["abi"].sparoa_expert_route(s["desc"], s["logits"], s["bias"], s["valid"], s["idx"],
                                 s["weights"], s["plan"], s["ws"])
    return s["idx"], s["weights"], s["views"]


def _own_experts(s):
    abi, c = s["abi"], s["case"]
    abi.sparoa_expert_plan(c["tokens"], c["top_k"], c["experts"], s["idx"], s["plan"],
                           s["plan_ws"])
    abi.sparoa_expert_ffn(s["desc"], s["act"], s["x"], s["w_up"], s["b_up"], s["w_down"],
                          s["b_down"], s["weights"], s["plan"], s["residual"], s["out"], s["ws"])
    return s["out"]


def _own_adapter(s):
    s["abi"].sparoa_fc_adapted(s["desc"], s["act"], s["x"], s["w"], s["bias"], s["a"], s["b"],
                               s["scale"], s["ids"], s["residual"], s["out"], s["ws"])
    return s["out"]


def _own_norm(s):
    s["abi"].sparoa_block_norm(s["desc"], s["y"], s["post_w"], s["post_b"], s["gate"], s["r"],
                               s["pre_w"], s["pre_b"], s["r_out"], s["n_out"])
    return s["r_out"], s["n_out"]


_OWN = dict(route=_own_route, experts=_own_experts, adapter=_own_adapter, norm=_own_norm)


def _plain_plan(idx, experts):
    """offsets [E + 1], order [T k] (slots by expert, -1 past the last), place [T k]."""
    flat = idx.reshape(-1)
    n = flat.numel()
    e = torch.where(flat < 0, experts, flat)
    order = torch.sort(e, stable=True).indices
    counts = torch.zeros(experts + 1, dtype=torch.int64, device=idx.device)
    counts.index_add_(0, e.long(), torch.ones_like(e, dtype=torch.int64))
    offsets = torch.zeros(experts + 1, dtype=torch.int64, device=idx.device)
    offsets[1:] = torch.cumsum(counts[:experts], 0)
    at = torch.arange(n, device=idx.device)
    place = torch.empty(n, dtype=torch.int64, device=idx.device)
    place[order] = at
    place = torch.where(flat < 0, -1, place)
    order = torch.where(at < offsets[experts], order, -1)
    return offsets.int(), order.int(), place.int()


def _plain_route(s):
    c = s["case"]
    low = float("-inf")
    l = s["logits"].float()
    ok = l > low
    if s["valid"] is not None:
        ok = ok & (s["valid"] != 0)[:, None]
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-l))
    else:
        top = torch.where(ok, l, low).amax(1, keepdim=True)
        ex = torch.where(ok, torch.exp(l - top), 0.0)
        score = ex / ex.sum(1, keepdim=True)
    # where only the order counts the logits have it
    key = l if s["bias"] is None and c["group_best"] == 1 else score
    if s["bias"] is not None:
        key = key + s["bias"]
    key = torch.where(ok, key, low)
    g = c["groups"]
    if g > 1:
        best = torch.sort(key.reshape(l.shape[0], g, -1), dim=2, descending=True).values
        best = best[:, :, :c["group_best"]]
        best = torch.where(best > low, best, 0.0).sum(2) + torch.where(best[:, :, 0] > low, 0.0, low)
        keep = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        in_group = torch.zeros_like(best, dtype=torch.bool).scatter_(1, keep, True)
        key = torch.where(in_group.repeat_interleave(l.shape[1] // g, 1), key, low)
    sel = torch.sort(key, dim=1, descending=True, stable=True)
    idx, got = sel.indices[:, :c["top_k"]], sel.values[:, :c["top_k"]] > low
    w = torch.where(got, score.gather(1, idx), 0.0)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    idx = torch.where(got, idx, -1).int()
    return idx, w * c["scale"], _plain_plan(idx, c["experts"])


def _act(v, name):
    if name == "silu":
        return v / (1.0 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * 0.5 ** 0.5))
    return torch.clamp(v, min=0.0) if name == "relu" else v


def _plain_experts(s):
    """The slots of every used expert, padded to the fullest, as batched products."""
    c = s["case"]
    k, h = c["top_k"], c["hidden"]
    offsets, order, place = (t.long() for t in _plain_plan(s["idx"], c["experts"]))
    counts = offsets[1:] - offsets[:-1]
    used = torch.nonzero(counts).reshape(-1)
    cap = int(counts.max())
    at = offsets[used][:, None] + torch.arange(cap, device=used.device)
    inside = torch.arange(cap, device=used.device) < counts[used][:, None]
    slot = order[torch.where(inside, at, 0)]
    xs = s["x"].float()[slot // k]                                     # [used, cap, hidden]
    u = torch.bmm(xs, s["w_up"][used].float().transpose(1, 2).contiguous())
    if s["b_up"] is not None:
        u = u + s["b_up"][used].float()[:, None]
    if c["gated"]:
        u = _act(u[:, :, :c["inner"]], c["act"]) * u[:, :, c["inner"]:]
    else:
        u = _act(u, c["act"])
    z = torch.bmm(u, s["w_down"][used].float().transpose(1, 2).contiguous())
    if s["b_down"] is not None:
        z = z + s["b_down"][used].float()[:, None]
    flat = torch.zeros(order.numel() + 1, h, device=z.device)           # the last row: no expert
    flat[at[inside]] = z[inside]
    out = (flat[place].reshape(-1, k, h) * s["weights"][:, :, None]).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return out.to(s["x"].dtype)


def _plain_adapter(s):
    c = s["case"]
    na, r = c["adapters"], c["rank"]
    x = s["x"].float()
    y = x @ s["w"].float().t()
    h = x @ s["a"].reshape(na * r, -1).float().t()
    mine = s["ids"][:, None] == torch.arange(na, device=x.device, dtype=torch.int32)
    h = h.reshape(-1, na, r) * (mine * s["scale"])[:, :, None]
    y = y + h.reshape(-1, na * r) @ s["b"].float().transpose(1, 2).reshape(na * r, -1)
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return _act(y, c["act"]).to(s["x"].dtype)


def _norm(v, kind, w, b):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    if kind != "none":
        v = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)
        v = v * w.to(v.dtype)
    return v if b is None else v + b.to(v.dtype)


def _plain_norm(s):
    c = s["case"]
    v = _norm(s["y"].float(), c["post"], s["post_w"], s["post_b"])
    if s["gate"] is not None:
        v = v * s["gate"].float().repeat_interleave(c["gate_rows"], 0)[:c["rows"]]
    r = c["c"] * s["r"].float() + v
    n = _norm(r, c["pre"], s["pre_w"], s["pre_b"])
    return r.to(s["r"].dtype), n.to(s["r"].dtype)


_PLAIN = dict(route=_plain_route, experts=_plain_experts, adapter=_plain_adapter, norm=_plain_norm)


# --------------------------------------------------------------- work, exact

def work(case):
    size = _SIZE[case["dtype"]]
    if case["kind"] == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        return dict(bytes=t * e * size + 4 * e * case["bias"] + 16 * t * k + 4 * e,
                    flops=4 * t * e)
    if case["kind"] == "experts":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        h, i = case["hidden"], case["inner"]
        mats = 3 if case["gated"] else 2
        live = t - int(case["pad"] * t)
        used = e * (1.0 - (1.0 - k / e) ** live)      # experts that some token chooses
        return dict(bytes=int(used * mats * h * i + t * h * (2 + case["residual"])) * size
                    + 8 * t * k, flops=2 * live * k * mats * h * i)
    if case["kind"] == "adapter":
        m, k, n, r = case["m"], case["k"], case["n"], case["rank"]
        na, req = case["adapters"], case["requests"] * (1.0 - case["bare"])
        used = na * (1.0 - (1.0 - 1.0 / na) ** req)   # adapters that some request names
        rows = m * (1.0 - case["bare"])
        return dict(bytes=int(m * k + n * k + m * n * (1 + case["residual"])
                              + used * r * (k + n)) * size + 4 * m,
                    flops=int(2 * m * k * n + 2 * rows * r * (k + n)))
    r, c = case["rows"], case["cols"]
    gates = -(-r // case["gate_rows"]) * case["gate"]
    return dict(bytes=(4 * r * c + gates * c + 2 * c) * size, flops=10 * r * c)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "route":
        return _exact_route(case, s)
    if kind == "experts":
        return _exact_experts(case, s)
    if kind == "adapter":
        x, w = s["x"].double(), s["w"].double()
        y = x @ w.t()
        for a in range(case["adapters"]):
            rows = (s["ids"] == a).nonzero().reshape(-1)
            if rows.numel():
                low = x[rows] @ s["a"][a].double().t()
                y[rows] += float(s["scale"][a]) * (low @ s["b"][a].double().t())
        for extra in ("bias", "residual"):
            if s[extra] is not None:
                y += s[extra].double()
        return y.clamp(min=0.0) if case["act"] == "relu" else y

    def normed(v, how, w, b):
        if how == "none":
            return v
        mean = v.mean(1, keepdim=True) if how == "layer" else torch.zeros_like(v[:, :1])
        var = ((v - mean) ** 2).sum(1, keepdim=True) / v.shape[1]
        v = (v - mean) * (var + 1e-6) ** -0.5 * w.double()
        return v if b is None else v + b.double()

    v = normed(s["y"].double(), case["post"], s["post_w"], s["post_b"])
    if s["gate"] is not None:
        of = torch.arange(case["rows"], device=v.device) // case["gate_rows"]
        v = v * s["gate"].double()[of]
    r = case["c"] * s["r"].double() + v
    return r, normed(r, case["pre"], s["pre_w"], s["pre_b"])


def _exact_route(case, s):
    l = s["logits"].double()
    t, e = l.shape
    alive = (l > float("-inf")).double()
    if s["valid"] is not None:
        alive = alive * s["valid"].double()[:, None]
    low = torch.full_like(l, float("-inf"))
    if case["score"] == "sigmoid":
        score = torch.sigmoid(l)
    else:
        score = torch.softmax(torch.where(alive > 0, l, low), 1)
    key = score if s["bias"] is None else score + s["bias"].double()
    key = torch.where(alive > 0, key, low)
    if case["groups"] > 1:
        per = e // case["groups"]
        top = torch.stack([key[:, i * per:(i + 1) * per].sort(1).values[:, -case["group_best"]:]
                           for i in range(case["groups"])], 1)
        total = torch.where(top == float("-inf"), torch.zeros_like(top), top).sum(2)
        total[(top == float("-inf")).all(2)] = float("-inf")
        kept = torch.sort(-total, dim=1, stable=True).indices[:, :case["top_groups"]]
        for i in range(case["groups"]):
            out = (kept != i).all(1)
            key[:, i * per:(i + 1) * per][out] = float("-inf")
    # equal keys in 64 bits: the lowest index
    picked = torch.sort(-key, dim=1, stable=True).indices[:, :case["top_k"]]
    there = key.gather(1, picked) > float("-inf")
    w = torch.where(there, score.gather(1, picked), torch.zeros_like(there, dtype=l.dtype))
    if case["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
    return None, w * case["scale"], None


def _exact_experts(case, s):
    if work(case)["flops"] > 1e12:
        return None
    x = s["x"].double()
    y = torch.zeros_like(x) if s["residual"] is None else s["residual"].double()
    for e in range(case["experts"]):
        tok, j = (s["idx"] == e).nonzero(as_tuple=True)
        if not tok.numel():
            continue
        u = x[tok] @ s["w_up"][e].double().t()
        if s["b_up"] is not None:
            u += s["b_up"][e].double()
        first = u[:, :case["inner"]]
        if case["act"] == "silu":
            v = first * torch.sigmoid(first)
        elif case["act"] == "gelu":
            v = first * 0.5 * torch.erfc(-first / 2.0 ** 0.5)
        else:
            v = first.clamp(min=0.0)
        if case["gated"]:
            v = v * u[:, case["inner"]:]
        z = v @ s["w_down"][e].double().t()
        if s["b_down"] is not None:
            z += s["b_down"][e].double()
        y.index_add_(0, tok, z * s["weights"][tok, j].double()[:, None])
    return y

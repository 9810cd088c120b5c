"""Routing to experts and the dispatch plan against a plain 64-bit routing in
numpy (token by token, from the definition).

Chosen experts must be equal: the test logits are multiples of 1/64 below 16,
so distinct logits, their scores and sums of two scores differ by far more
than fp32 rounding (biases are multiples of 1/4 that keep them apart or equal
logits equal), and equal ones tie to the lowest index on both sides.  Weights:
fp32 exponentials, quotients and sums of at most 512 terms, 64 roundings of
2^-24 relative."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

RTOL = 64 * 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _abi():
    from paper_2511_19457_amd import abi
    return abi


def reference(l, k, score, groups, top_groups, best, bias, renorm, scale, mask):
    t_, e_ = l.shape
    idx, w = np.full((t_, k), -1, np.int32), np.zeros((t_, k))
    for t in range(t_):
        ok = [e for e in range(e_) if l[t, e] > -np.inf and (mask is None or mask[t])]
        if not ok:
            continue
        if score == 0:
            top = max(l[t, e] for e in ok)
            x = {e: 1.0 if l[t, e] == top else float(np.exp(l[t, e] - top)) for e in ok}
            total = sum(x.values())
            s = {e: x[e] / total for e in ok}
        else:
            s = {e: 1.0 / (1.0 + np.exp(-l[t, e])) for e in ok}
        # the order of the logits where nothing is added to the scores
        plain = bias is None and (groups == 1 or best == 1)
        # (keys are fp32 by definition: scores the sum cannot tell apart tie)
        key = {e: l[t, e] if plain else np.float32(s[e]) + np.float32(0 if bias is None
                                                                      else bias[e]) for e in ok}
        key = {e: v for e, v in key.items() if v > -np.inf}
        if groups > 1:
            per = e_ // groups
            gs = []
            for g in range(groups):
                mine = sorted((v for e, v in key.items() if e // per == g), reverse=True)[:best]
                if mine:
                    gs.append((-sum(mine), g))
            kept = {g for _, g in sorted(gs)[:top_groups]}
            key = {e: v for e, v in key.items() if e // per in kept}
        chosen = sorted(key, key=lambda e: (-key[e], e))[:k]
        if score == 0 and renorm and chosen:
            top = max(l[t, e] for e in chosen)
            s = {e: 1.0 if l[t, e] == top else float(np.exp(l[t, e] - top)) for e in chosen}
        total = sum(s[e] for e in chosen) if renorm else 1.0
        for j, e in enumerate(chosen):
            idx[t, j], w[t, j] = e, (s[e] / total if total > 0 else 0.0) * scale
    return idx, w


def check_plan(plan, idx, t, k, e):
    """The plan against its definition, from the choices the call gave."""
    offsets, order, place = (v.cpu().numpy() for v in _abi().expert_plan_views(plan, t, k, e))
    flat = idx.reshape(-1)
    live = (flat >= 0) & (flat < e)
    by = np.where(live, flat, e)
    want = np.argsort(by, kind="stable").astype(np.int64)
    counts = np.bincount(by, minlength=e + 1)[:e]
    assert np.array_equal(offsets, np.concatenate([[0], np.cumsum(counts)]))
    n = int(counts.sum())
    assert np.array_equal(order[:n], want[:n]) and (order[n:] == -1).all()
    back = np.full(flat.size, -1)
    back[want[:n]] = np.arange(n)
    assert np.array_equal(place, back)
    active = plan.cpu().numpy()[e + 1:2 * e + 2]
    ids = np.nonzero(counts)[0]
    assert active[0] == ids.size and np.array_equal(active[1:1 + ids.size], ids)


def logits(t, e, dt, seed):
    g = np.random.default_rng(seed)
    v = g.integers(-512, 512, (t, e)) / 64.0
    return torch.from_numpy(np.clip(v, -8, 7.9375)).to(DT[dt])


def run(l, k, score=0, groups=1, top_groups=1, best=1, bias=None, renorm=False, scale=1.0,
        mask=None):
    abi, dev = _abi(), torch.device("cuda")
    t, e = l.shape
    d = abi.expert_route_desc(t, e, k, l.dtype, score=score, groups=groups, top_groups=top_groups,
                              group_best=best, renormalise=renorm, scale=scale)
    idx = torch.full((t, k), 99, dtype=torch.int32, device=dev)
    w = torch.full((t, k), 99.0, device=dev)
    plan = torch.full((abi.sparoa_expert_plan_words(t, k, e),), 99, dtype=torch.int32, device=dev)
    ws = torch.empty(abi.sparoa_expert_route_workspace_size(d), dtype=torch.uint8, device=dev)
    on = lambda v: None if v is None else torch.as_tensor(v).to(dev)
    args = (d, l.to(dev), on(bias), on(mask), idx, w)
    abi.sparoa_expert_route(*args, plan, ws)
    torch.cuda.synchronize()
    got = idx.cpu().numpy(), w.cpu().numpy(), plan.clone()
    # the plan of the same choices, and routing alone
    plan.fill_(99)
    abi.sparoa_expert_plan(t, k, e, idx, plan, torch.empty(
        abi.sparoa_expert_plan_workspace_size(t, k, e), dtype=torch.uint8, device=dev))
    check_plan(plan, got[0], t, k, e)
    idx.fill_(99)
    w.fill_(99)
    abi.sparoa_expert_route(*args)
    assert np.array_equal(idx.cpu().numpy(), got[0]) and np.array_equal(w.cpu().numpy(), got[1])
    return got


def check(l, k, **kw):
    idx, w, plan = run(l, k, **kw)
    mask = kw.get("mask")
    ri, rw = reference(l.double().numpy(), k, kw.get("score", 0), kw.get("groups", 1),
                       kw.get("top_groups", 1), kw.get("best", 1), kw.get("bias"),
                       kw.get("renorm", False), kw.get("scale", 1.0), mask)
    assert np.array_equal(idx, ri), np.argwhere(idx != ri)[:5]
    assert np.all(np.abs(w - rw) <= RTOL * np.abs(rw) + 1e-37), np.abs(w - rw).max()
    check_plan(plan, idx, l.shape[0], k, l.shape[1])


# tokens x experts, choices: one token; around 64 tokens (one work-group) and
# its next; odd sizes; experts around every lane layout
SIZES = [(1, 1, 1), (1, 64, 8), (3, 60, 4), (64, 65, 6), (65, 128, 2), (130, 129, 3), (257, 8, 8),
         (63, 256, 8), (1003, 257, 5), (40, 512, 32), (4500, 40, 2)]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("score,renorm", [(0, False), (0, True), (1, False), (1, True)])
def test_sizes(dt, size, score, renorm):
    t, e, k = size
    check(logits(t, e, dt, SIZES.index(size)), k, score=score, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("groups,top_groups,best", [(2, 1, 1), (8, 4, 2), (5, 3, 2), (64, 7, 1),
                                                    (4, 4, 2), (12, 2, 1)])
@pytest.mark.parametrize("per", [1, 3, 8])
def test_groups(groups, top_groups, best, per):
    e = groups * per
    k = min(4, per * top_groups)
    for score in (0, 1):
        check(logits(37, e, "f32", groups + per), k, score=score, groups=groups,
              top_groups=top_groups, best=best, renorm=True)


@pytest.mark.parametrize("score", [0, 1])
def test_bias_chooses_and_joins_no_weight(score):
    g = np.random.default_rng(5)
    bias = (g.integers(-8, 9, 48) / 4.0).astype(np.float32)
    check(logits(90, 48, "f32", 70), 6, score=score, bias=bias, renorm=True)
    bias[3], bias[7] = -np.inf, np.nan
    check(logits(90, 48, "f16", 71), 6, score=score, bias=bias, groups=6, top_groups=2, best=2)


def test_masked_tokens_and_experts():
    l = logits(200, 30, "f32", 80)
    mask = (np.arange(200) % 3 != 0).astype(np.uint8) * 255
    l[:, 4] = float("-inf")
    l[5:9] = float("-inf")                       # no expert left
    l[10, 1:] = float("-inf")                    # one left
    l[11] = float("nan")
    l[13, ::2] = float("nan")
    for score in (0, 1):
        for renorm in (False, True):
            check(l, 5, score=score, renorm=renorm, mask=mask)
            check(l, 4, score=score, renorm=renorm, groups=5, top_groups=2, best=2)
    check(l, 5, mask=np.zeros(200, np.uint8))    # nothing is routed


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_lowest_values_ties_and_infinities(dt):
    l = logits(12, 24, dt, 90)
    low = torch.finfo(DT[dt]).min
    l[0] = low                                   # a row of the type's lowest value: all equal
    l[1, 5:] = low
    l[2] = 0
    l[3, 20] = float("inf")
    l[4, [2, 19, 3]] = float("inf")
    for renorm in (False, True):
        check(l, 6, score=0, renorm=renorm)
    l[1, 5:] = -8                                # (a score of 0 ties with its like)
    l[0] = -8
    check(l, 6, score=1, renorm=True)


def test_far_below_the_largest_logit():
    """Choices kept to a group far below the row's best keep their ratios."""
    l = torch.full((2, 8), -200.0)
    l[:, 4:] = torch.tensor([-201.0, -199.0, -200.0, -203.0])
    l[:, 0] = 100.0
    bias = np.array([-9, -9, -9, -9, 9, 9, 9, 9], np.float32)
    idx, w, _ = run(l, 2, score=0, groups=2, top_groups=1, bias=bias, renorm=True)
    assert set(idx[0]) <= {4, 5, 6, 7}
    x = np.exp(l[0].numpy()[idx[0]].astype(np.float64) - l[0].numpy()[idx[0]].max())
    assert np.allclose(w[0], x / x.sum(), rtol=1e-6)


@pytest.mark.parametrize("t,k", [(1, 1), (50, 3), (4096, 1), (4097, 1), (9000, 7), (70000, 2)])
def test_plan_of_given_choices(t, k):
    """Uneven choices, values that are no expert, an expert chosen twice by a token."""
    abi, dev = _abi(), torch.device("cuda")
    g = np.random.default_rng(t)
    e = 100
    idx = np.minimum(g.geometric(0.05, (t, k)) - 1, e + 3).astype(np.int32)
    idx[g.random((t, k)) < 0.1] = -1
    idx[g.random((t, k)) < 0.01] = np.iinfo(np.int32).min
    ws = torch.empty(abi.sparoa_expert_plan_workspace_size(t, k, e), dtype=torch.uint8, device=dev)
    plan = torch.full((abi.sparoa_expert_plan_words(t, k, e),), 99, dtype=torch.int32, device=dev)
    abi.sparoa_expert_plan(t, k, e, torch.from_numpy(idx).to(dev), plan, ws)
    check_plan(plan, idx, t, k, e)

"""The experts' products (sparoa_expert_ffn) against their formula in 64-bit
numpy, expert by expert.

Tolerance, by propagation: fp32 products are within 1e-5 of their sums of
absolute terms (the framework's fp32 bound), activations have slopes of at
most 1.13, u and each slot's down product are rounded to the dtype once
(u = 2^-8, 2^-11, 2^-24) and so is the result; subnormal results may be off by
a step of the dtype."""
import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -24, "f32": 2.0 ** -149}
SUM, SLOPE = 1e-5, 1.13


def _abi():
    from paper_2511_19457_amd import abi
    return abi


def _act(v, name):
    if name == "silu":
        return v / (1.0 + np.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(torch.from_numpy(v) * 0.5 ** 0.5).numpy())
    if name == "none":
        return v
    return np.clip(v, 0.0, 6.0 if name == "relu6" else np.inf)


def reference(x, w_up, b_up, w_down, b_down, idx, weights, residual, gated, act, dt):
    """(y, its absolute error bound)."""
    n = lambda t: None if t is None else t.double().numpy()
    x, w_up, b_up, w_down, b_down, residual = map(n, (x, w_up, b_up, w_down, b_down, residual))
    y = np.zeros(x.shape) if residual is None else residual.copy()
    err = SUM * np.abs(y)
    inner = w_down.shape[2]
    for e in range(w_up.shape[0]):
        tok, j = np.nonzero(idx == e)
        if not tok.size:
            continue
        pre, size = x[tok] @ w_up[e].T, np.abs(x[tok]) @ np.abs(w_up[e]).T
        if b_up is not None:
            pre, size = pre + b_up[e], size + np.abs(b_up[e])
        v, verr = _act(pre[:, :inner], act), SLOPE * SUM * size[:, :inner]
        if gated:
            up, uerr = pre[:, inner:], SUM * size[:, inner:]
            v, verr = v * up, verr * (np.abs(up) + uerr) + np.abs(v) * uerr
        verr = verr + (U[dt] + SUM) * (np.abs(v) + verr) + TINY[dt]
        z = v @ w_down[e].T
        zerr = verr @ np.abs(w_down[e]).T + SUM * (np.abs(v) @ np.abs(w_down[e]).T)
        if b_down is not None:
            z, zerr = z + b_down[e], zerr + SUM * np.abs(b_down[e])
        zerr = zerr + U[dt] * (np.abs(z) + zerr) + TINY[dt]
        w = weights[tok, j].astype(np.float64)[:, None]
        np.add.at(y, tok, w * z)
        np.add.at(err, tok, np.abs(w) * (zerr + SUM * np.abs(z)))
    return y, err + U[dt] * (np.abs(y) + err) + TINY[dt]


def choices(t, k, e, kind, seed):
    g = np.random.default_rng(seed)
    idx = np.stack([g.permutation(e)[:k] for _ in range(t)]).astype(np.int32)
    if kind == "one":                    # every token's first choice is the last expert
        idx = np.where(idx == e - 1, idx[:, :1], idx)
        idx[:, 0] = e - 1
    if kind == "padded":
        idx[g.random((t, k)) < 0.3] = -1
        idx[t // 2] = -1                 # a token without experts
    if kind == "empty":
        idx[:] = -1
    return idx


def run(t, e, k, hidden, inner, dt, gated, act, kind="even", bias=False, residual=False, seed=0,
        in_place=False, poison=False):
    abi, dev = _abi(), torch.device("cuda")
    up = 2 * inner if gated else inner
    mk = lambda shape, i, std: synth.normal(shape, dt, 8000 + 20 * seed + i, std=std)
    x = mk((t, hidden), 0, 1.0)
    w_up, w_down = mk((e, up, hidden), 1, (2 / hidden) ** 0.5), mk((e, hidden, inner), 2,
                                                                  inner ** -0.5)
    b_up, b_down = (mk((e, up), 3, 0.3), mk((e, hidden), 4, 0.3)) if bias else (None, None)
    res = mk((t, hidden), 5, 1.0) if residual else None
    idx = choices(t, k, e, kind, seed)
    weights = np.random.default_rng(seed + 1).random((t, k)).astype(np.float32)
    if poison:                           # masked places: their weights, and unused experts
        weights[idx < 0] = np.nan
        for u in range(e):
            if not (idx == u).any():
                w_up[u], w_down[u] = float("nan"), float("inf")
    ref, err = reference(x, w_up, b_up, w_down, b_down, idx, weights, res, gated, act, dt)
    on = lambda v: None if v is None else v.to(dev)
    res_d = on(res)
    y = res_d if in_place else torch.full((t, hidden), float("nan"), dtype=DT[dt], device=dev)
    d = abi.expert_ffn_desc(t, k, e, hidden, inner, DT[dt], gated=gated, has_bias=bias)
    plan = torch.empty(abi.sparoa_expert_plan_words(t, k, e), dtype=torch.int32, device=dev)
    abi.sparoa_expert_plan(t, k, e, torch.from_numpy(idx).to(dev), plan, torch.empty(
        abi.sparoa_expert_plan_workspace_size(t, k, e), dtype=torch.uint8, device=dev))
    ws = torch.full((abi.sparoa_expert_ffn_workspace_size(d),), 255, dtype=torch.uint8, device=dev)
    code = getattr(abi, "ACT_" + act.upper())
    abi.sparoa_expert_ffn(d, code, on(x), on(w_up), on(b_up), on(w_down), on(b_down),
                          torch.from_numpy(weights).to(dev), plan, res_d, y, ws)
    got = y.double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= err)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3],
                           ref[bad][:3], err[bad][:3])
    return y


# tokens, experts, choices, hidden, inner: one token; widths around a step of
# K (64), odd ones, rows that start off 16 bytes; segments of 1 to some hundred
# rows; a hundred and more rows an expert at the end
SHAPES = [(1, 8, 2, 64, 64), (1, 1, 1, 8, 8), (3, 5, 2, 72, 40), (16, 4, 1, 128, 96),
          (17, 3, 3, 200, 33), (33, 2, 2, 33, 200), (50, 64, 8, 136, 8), (65, 2, 1, 1, 1),
          (70, 6, 2, 768, 264), (130, 3, 2, 260, 136), (300, 2, 2, 192, 320), (517, 4, 2, 320, 256),
          (700, 3, 1, 64, 1000), (257, 5, 3, 1000, 72),
          (2100, 16, 1, 64, 1100), (2100, 16, 1, 1096, 72)]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("gated", [False, True])
def test_shapes(dt, shape, gated):
    i = SHAPES.index(shape)
    run(*shape, dt, gated, ("silu", "gelu", "relu")[i % 3], bias=i % 2 == 0, residual=i % 3 == 0,
        seed=i)


@pytest.mark.parametrize("kind", ["one", "padded", "empty"])
@pytest.mark.parametrize("shape", [(40, 8, 2, 128, 72), (400, 8, 2, 128, 136), (90, 30, 4, 50, 30),
                                   (600, 4, 3, 256, 128)])
@pytest.mark.parametrize("gated", [False, True])
def test_uneven_and_masked_choices(kind, shape, gated):
    run(*shape, "bf16", gated, "silu", kind=kind, bias=True, residual=True, poison=True, seed=40)
    run(*shape, "f16", gated, "none", kind=kind, seed=41)


@pytest.mark.parametrize("act", ["none", "relu", "relu6", "silu", "gelu"])
def test_activations(act):
    run(20, 4, 2, 96, 64, "f32", False, act, seed=50)
    run(200, 2, 2, 96, 128, "bf16", True, act, seed=51)


def test_residual_in_place_and_repeats():
    a = run(300, 6, 2, 256, 128, "bf16", True, "silu", residual=True, in_place=True, seed=60)
    b = run(300, 6, 2, 256, 128, "bf16", True, "silu", residual=True, seed=60)
    assert torch.equal(a, b)             # the same sums in the same order


def test_in_a_graph():
    """Captured with its plan, replayed over changed inputs."""
    abi, dev = _abi(), torch.device("cuda")
    t, e, k, h, i = 48, 8, 2, 128, 64
    x = torch.empty(t, h, dtype=torch.bfloat16, device=dev)
    w_up = synth.normal((e, 2 * i, h), "bf16", 9001, std=0.1).to(dev)
    w_down = synth.normal((e, h, i), "bf16", 9002, std=0.1).to(dev)
    logits = torch.empty(t, e, device=dev)
    idx = torch.empty(t, k, dtype=torch.int32, device=dev)
    weights = torch.empty(t, k, device=dev)
    plan = torch.empty(abi.sparoa_expert_plan_words(t, k, e), dtype=torch.int32, device=dev)
    rd = abi.expert_route_desc(t, e, k, torch.float32, renormalise=True)
    fd = abi.expert_ffn_desc(t, k, e, h, i, torch.bfloat16, gated=True)
    rws = torch.empty(abi.sparoa_expert_route_workspace_size(rd), dtype=torch.uint8, device=dev)
    fws = torch.empty(abi.sparoa_expert_ffn_workspace_size(fd), dtype=torch.uint8, device=dev)
    y = torch.empty(t, h, dtype=torch.bfloat16, device=dev)

    def step():
        abi.sparoa_expert_route(rd, logits, None, None, idx, weights, plan, rws)
        abi.sparoa_expert_ffn(fd, abi.ACT_SILU, x, w_up, None, w_down, None, weights, plan, None,
                              y, fws)

    x.copy_(synth.normal((t, h), "bf16", 9003))
    logits.copy_(synth.normal((t, e), "f32", 9004))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(4):
        x.copy_(synth.normal((t, h), "bf16", 9010 + rep))
        logits.copy_(synth.normal((t, e), "f32", 9020 + rep))
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        replayed = y.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(replayed, y) and y.abs().sum() > 0

"""FCs with low-rank adapters of many requests (sparoa_fc_adapted) against the
formula in 64-bit numpy, adapter by adapter.

Tolerance: fp32 products within 1e-5 of their sums of absolute terms; a_a x is
rounded at most once to the dtype (u = 2^-8, 2^-11, 2^-24), the result once."""
import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -24, "f32": 2.0 ** -149}
SUM = 1e-5


def _abi():
    from paper_2511_19457_amd import abi
    return abi


def reference(x, w, bias, a, b, scale, ids, residual, act, dt):
    n = lambda t: None if t is None else t.double().numpy()
    x, w, bias, a, b, residual = map(n, (x, w, bias, a, b, residual))
    y, err = x @ w.T, SUM * (np.abs(x) @ np.abs(w).T)
    for i in range(a.shape[0]):
        rows = np.nonzero(ids == i)[0]
        if not rows.size:
            continue
        s = float(scale[i])
        h, herr = s * (x[rows] @ a[i].T), abs(s) * SUM * (np.abs(x[rows]) @ np.abs(a[i]).T)
        herr = herr + (U[dt] + SUM) * (np.abs(h) + herr) + TINY[dt]
        y[rows] += h @ b[i].T
        err[rows] += herr @ np.abs(b[i]).T + SUM * (np.abs(h) @ np.abs(b[i]).T)
    for extra in (bias, residual):
        if extra is not None:
            y = y + extra
            err = err + SUM * np.abs(extra)
    if act:
        y = np.clip(y, 0.0, 6.0 if act == 2 else np.inf)
    return y, err + U[dt] * (np.abs(y) + err) + TINY[dt]


def run(m, k, n, adapters, rank, dt, kind="runs", act=0, bias=False, residual=False, seed=0,
        in_place=False, poison=False):
    abi, dev = _abi(), torch.device("cuda")
    g = np.random.default_rng(seed)
    mk = lambda shape, i, std: synth.normal(shape, dt, 9100 + 20 * seed + i, std=std)
    x, w = mk((m, k), 0, 1.0), mk((n, k), 1, k ** -0.5)
    a, b = mk((adapters, rank, k), 2, k ** -0.5), mk((adapters, n, rank), 3, 0.7)
    bv = mk((n,), 4, 0.3) if bias else None
    res = mk((m, n), 5, 1.0) if residual else None
    scale = (g.random(adapters) + 0.5).astype(np.float32)
    if kind == "runs":                   # requests of several rows
        ids = np.sort(g.integers(-1, adapters, m))[::-1].copy()
    elif kind == "mixed":                # every row its own
        ids = g.integers(-2, adapters + 2, m)
    elif kind == "none":
        ids = np.where(g.random(m) < 0.5, -1, adapters)
    else:
        ids = np.zeros(m, np.int64)
    ids = ids.astype(np.int32)
    if poison:                           # adapters that no row names
        for i in range(adapters):
            if not (ids == i).any():
                a[i], b[i], scale[i] = float("nan"), float("inf"), np.nan
    ref, err = reference(x, w, bv, a, b, scale, ids, res, act, dt)
    on = lambda v: None if v is None else v.to(dev)
    res_d = on(res)
    y = res_d if in_place else torch.full((m, n), float("nan"), dtype=DT[dt], device=dev)
    d = abi.fc_adapted_desc(m, k, n, adapters, rank, DT[dt], has_bias=bias)
    ws = torch.full((abi.sparoa_fc_adapted_workspace_size(d),), 255, dtype=torch.uint8, device=dev)
    abi.sparoa_fc_adapted(d, act, on(x), on(w), on(bv), on(a), on(b),
                          torch.from_numpy(scale).to(dev), torch.from_numpy(ids).to(dev), res_d, y,
                          ws)
    got = y.double().cpu().numpy()
    bad = ~(np.abs(got - ref) <= err)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3],
                           ref[bad][:3], err[bad][:3])
    return y


# m, k, n, adapters, rank: single rows, decode batches, odd widths and ranks,
# rows that start off 16 bytes, several hundred rows, ranks above a step of K
SHAPES = [(1, 64, 64, 1, 8), (1, 8, 1, 3, 1), (5, 200, 130, 4, 16), (16, 1000, 72, 16, 4),
          (33, 33, 47, 5, 3), (64, 256, 512, 40, 32), (65, 520, 264, 3, 64), (130, 96, 1000, 2, 24),
          (333, 768, 100, 9, 8), (300, 1001, 64, 2, 100), (700, 256, 384, 12, 136),
          (1030, 128, 520, 70, 16), (2050, 320, 1024, 5, 40), (2050, 200, 2104, 70, 12),
          (6200, 64, 2056, 9, 20)]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["runs", "mixed"])
def test_shapes(dt, shape, kind):
    i = SHAPES.index(shape)
    run(*shape, dt, kind=kind, act=i % 3, bias=i % 2 == 0, residual=i % 3 == 1, seed=i)


@pytest.mark.parametrize("kind", ["none", "same", "runs"])
@pytest.mark.parametrize("m", [7, 64, 500, 2500])
def test_unused_adapters_are_not_read(kind, m):
    run(m, 256, 320, 6 if kind != "runs" else 2 * m, 16, "bf16", kind=kind, poison=True, seed=30)


def test_residual_in_place_and_repeats():
    for m in (40, 1500):
        a = run(m, 256, 256, 5, 16, "f16", kind="mixed", residual=True, in_place=True, seed=31)
        b = run(m, 256, 256, 5, 16, "f16", kind="mixed", residual=True, seed=31)
        assert torch.equal(a, b)

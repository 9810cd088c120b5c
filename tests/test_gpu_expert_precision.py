"""What the experts' products promise of their roundings (sparoa_expert_ffn).

u is made exact here (each row of w_up copies one feature of x, no activation),
so that a down product's error is its fp32 sum's and its own rounding's.  The
residual is minus the exact output rounded to the dtype: what is left over is
some 2^-8 of the output, and its last rounding hides nothing.

Tolerance of a down product z, its terms' absolute sum s: fp32 sums 1e-5 s (the
framework's bound), 2^-10 |z| where it goes to the weighted sum as 9 bits behind
the point (bf16, many rows, top_k > 1), and 2^-38 of the largest of its 8 channels
where that is more (half of a subnormal fp16's last bit but one, 2^-24, where the
largest is 2^14 or more).  The weighted sum and the residual add 1e-5
of their terms, the result one rounding of what is left."""
import numpy as np
import pytest
import torch

import synth
from tests import test_gpu_expert_ffn as ffn

pytestmark = pytest.mark.gpu

DT, U, TINY, SUM = ffn.DT, ffn.U, ffn.TINY, ffn.SUM


def call(x, w_up, w_down, idx, weights, residual=None, act="none", gated=False):
    from paper_2511_19457_amd import abi
    dev = torch.device("cuda")
    t, k, e = x.shape[0], idx.shape[1], w_up.shape[0]
    d = abi.expert_ffn_desc(t, k, e, x.shape[1], w_down.shape[2], x.dtype, gated=gated)
    plan = torch.empty(abi.sparoa_expert_plan_words(t, k, e), dtype=torch.int32, device=dev)
    abi.sparoa_expert_plan(t, k, e, torch.from_numpy(idx).to(dev), plan, torch.empty(
        abi.sparoa_expert_plan_workspace_size(t, k, e), dtype=torch.uint8, device=dev))
    ws = torch.full((abi.sparoa_expert_ffn_workspace_size(d),), 255, dtype=torch.uint8, device=dev)
    y = torch.full_like(x, float("nan"), device=dev)
    abi.sparoa_expert_ffn(d, getattr(abi, "ACT_" + act.upper()), x.to(dev), w_up.to(dev), None,
                          w_down.to(dev), None, torch.from_numpy(weights).to(dev), plan,
                          None if residual is None else residual.to(dev), y, ws)
    return y.double().cpu().numpy()


def copies(e, inner, hidden, dt, seed):
    """w_up [e, inner, hidden] whose rows pick one feature each, and which."""
    pick = np.random.default_rng(seed).integers(0, hidden, (e, inner))
    w = torch.zeros(e, inner, hidden, dtype=DT[dt])
    w.scatter_(2, torch.from_numpy(pick)[:, :, None], 1.0)
    return w, pick


def left_over(t, e, k, hidden, inner, dt, seed, scaled=False, channels=None):
    """(what the call leaves, what it should, its bound, the exact output)."""
    x = synth.normal((t, hidden), dt, 9970 + seed)
    w_up, pick = copies(e, inner, hidden, dt, seed)
    w_down = synth.normal((e, hidden, inner), "f32", 9980 + seed, std=inner ** -0.5)
    if channels is not None:
        w_down *= channels[:, None]
    w_down = w_down.to(DT[dt])
    idx = ffn.choices(t, k, e, "even", seed)
    weights = (np.random.default_rng(seed).random((t, k)) + 0.5).astype(np.float32)
    xs, wd = x.double().numpy(), w_down.double().numpy()
    y, err = np.zeros((t, hidden)), np.zeros((t, hidden))
    for i in range(e):
        tok, j = np.nonzero(idx == i)
        u, w = xs[tok][:, pick[i]], weights[tok, j].astype(np.float64)[:, None]
        z, s = u @ wd[i].T, np.abs(u) @ np.abs(wd[i]).T
        np.add.at(y, tok, w * z)
        own = 2 * SUM * s
        if scaled:
            size = np.abs(np.pad(z, ((0, 0), (0, -hidden % 8)))).reshape(len(tok), -1, 8)
            top = np.repeat(size.max(2), 8, 1)[:, :hidden]
            own += np.maximum(2.0 ** -10 * np.abs(z), 2.0 ** -38 * top)
        np.add.at(err, tok, w * own)
    residual = torch.from_numpy(-y).to(DT[dt])
    want = y + residual.double().numpy()
    err += SUM * np.abs(y)
    got = call(x, w_up, w_down, idx, weights, residual)
    return got, want, err + U[dt] * (np.abs(want) + err) + TINY[dt], y


# tokens, experts, choices, hidden, inner: few rows and many, whole vectors and not
@pytest.mark.parametrize("dt,shape", [
    ("bf16", (10, 8, 2, 128, 64)), ("bf16", (20, 8, 2, 131, 61)), ("f16", (10, 8, 2, 128, 64)),
    ("f16", (600, 4, 2, 128, 64)), ("f16", (600, 4, 2, 131, 61)), ("bf16", (600, 4, 1, 128, 64)),
    ("bf16", (600, 4, 1, 131, 61)), ("f32", (60, 4, 2, 128, 64)), ("f32", (600, 4, 2, 131, 61))])
def test_down_products_stay_fp32(dt, shape):
    got, want, bound, _ = left_over(*shape, dt, 1)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())


SCALED = [(600, 4, 2, 128, 64), (600, 4, 2, 131, 61), (3000, 8, 8, 256, 64)]


@pytest.mark.parametrize("shape", SCALED)
def test_scaled_down_products_round_once_without_bias(shape):
    """Each within half of its last bit, and all of them together as often up as
    down: 10^5 and more roundings of 2^-10 / sqrt 3 at most move the sum by less
    than 1e-5 of itself (5 deviations)."""
    got, want, bound, y = left_over(*shape, "bf16", 2, scaled=True)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())
    gain = ((got - want) * y).sum() / (y * y).sum()
    assert abs(gain) < 5 * 2.0 ** -10 / 3 ** 0.5 / y.size ** 0.5 + 1e-6, gain


@pytest.mark.parametrize("shape", SCALED[:2])
@pytest.mark.parametrize("power", [-90, 0, 60])
def test_scaled_channels_of_unlike_size(shape, power):
    """Channels 2^26 below their neighbours have their 9 bits too."""
    down = 2.0 ** np.array([0.0, -20.0, -10.0, -26.0, 0.0, -17.0, -24.0, -22.0])
    channels = torch.from_numpy(np.resize(down, shape[3]) * 2.0 ** power).float()
    got, want, bound, _ = left_over(*shape, "bf16", 3, scaled=True, channels=channels)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), "all ones",
                                   "all ones, negative"])
def test_scaled_neighbours_of_an_infinity_or_nan(value):
    """Channels of one number each (z = x[0] w), so that what stands beside the
    infinity or NaN is exact: large, small and ordinary ones keep their bits."""
    t, e, k, hidden, inner = 200, 2, 2, 64, 64
    x = torch.ones(t, hidden, dtype=torch.bfloat16)
    w_up = torch.zeros(e, inner, hidden, dtype=torch.bfloat16)
    w_up[:, 0, 0] = 1.0
    rows = torch.tensor([1.0, 1e5, -7e4, 1e-3, 1.5, -1e5, 98304.0, 0.01]).repeat(hidden // 8)
    rows[8:16] *= 2.0 ** -60
    rows[16:24] = torch.tensor([1e-8, 2e-8, -3e-8, 0.0, 5e-8, 1e-8, 1e-8, 1e-8])
    rows[24:32] *= 2.0 ** 100
    w_down = torch.zeros(e, hidden, inner, dtype=torch.bfloat16)
    w_down[:, :, 0] = rows.to(torch.bfloat16)
    at = torch.arange(hidden) % 8 == torch.arange(hidden) // 8      # one channel of each block
    if isinstance(value, str):
        w_down.view(torch.int16)[1, at, 0] = 0x7FFF if value == "all ones" else -1
    else:
        w_down[1, at, 0] = value
    idx = np.tile(np.array([[0, 1]], np.int32), (t, 1))
    weights = np.full((t, k), 0.5, np.float32)
    got = call(x, w_up, w_down, idx, weights)
    want = w_down[0, :, 0].double().numpy()           # 0.5 z + 0.5 z, bf16 numbers: exact
    at = at.numpy()
    assert np.array_equal(got[:, ~at], np.tile(want[~at], (t, 1)))
    if not isinstance(value, str) and value == value:
        assert (got[:, at] == value).all()
    else:
        assert np.isnan(got[:, at]).all()


def test_scaled_numbers_next_to_the_largest_stay_finite():
    t, e, k, hidden, inner = 200, 2, 2, 64, 64
    x = torch.ones(t, hidden, dtype=torch.bfloat16)
    w_up = torch.zeros(e, inner, hidden, dtype=torch.bfloat16)
    w_up[:, 0, 0] = w_up[:, 1, 1] = 1.0
    w_down = torch.zeros(e, hidden, inner, dtype=torch.bfloat16)
    most = torch.tensor(float(2 ** 128 - 2 ** 120), dtype=torch.float64)
    w_down[:, :, 0] = most.to(torch.bfloat16)
    w_down[:, :, 1] = 0.998 * 2.0 ** 120              # z within 2^-17 of 2^128
    w_down[:, 1::2] *= -1
    idx = np.tile(np.array([[0, 1]], np.int32), (t, 1))
    got = call(x, w_up, w_down, idx, np.full((t, k), 0.25, np.float32))
    z = w_down[0, :, :2].double().sum(1).numpy()
    assert np.isfinite(got).all() and (np.abs(got - 0.5 * z) <= 2.0 ** -8 * np.abs(z)).all()


# ---------------------------------------------------------------- activations

def _through(v, act, dt, hidden, rows):
    """act(v): both matrices the identity, one expert of `rows` rows a token."""
    t = -(-len(v) // hidden)
    t = max(t, rows)
    x = torch.zeros(t * hidden, dtype=DT[dt])
    x[:len(v)] = v
    eye = torch.eye(hidden, dtype=DT[dt])[None]
    got = call(x.reshape(t, hidden), eye, eye, np.zeros((t, 1), np.int32),
               np.ones((t, 1), np.float32), act=act)
    return got.reshape(-1)[:len(v)]


# (few rows and many; whole vectors, and rows that start off 16 bytes)
@pytest.mark.parametrize("hidden,rows", [(64, 1), (64, 300), (61, 1), (61, 300)])
def test_silu_fp32(hidden, rows):
    """exp to one unit in the last place (two halves), the sum and the division to
    half of one: 4 2^-24, and a second-order rest."""
    v = torch.cat([torch.linspace(-60, 30, 3001), torch.linspace(-1e-3, 1e-3, 101)])
    got, w = _through(v, "silu", "f32", hidden, rows), v.double().numpy()
    want = w / (1.0 + np.exp(-w))
    off = np.abs(got - want) / np.maximum(np.abs(want), 2.0 ** -126)
    assert off.max() <= 4.5 * 2.0 ** -24, (off.max() * 2 ** 24, v[off.argmax()])


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("hidden,rows", [(64, 1), (64, 300), (61, 1), (61, 300)])
def test_gelu_tail(dt, hidden, rows):
    """Far below 0, where 1 + erf would cancel: the argument v / sqrt 2 is off by 2
    roundings, which v^2 + 1 times as many in the result follow; erfc to 16 units in
    the last place; two products."""
    import math
    v = torch.linspace(-9.5 if dt == "f32" else -5.0, 4.0, 2001).to(DT[dt])
    got, w = _through(v, "gelu", dt, hidden, rows), v.double().numpy()
    want = np.array([0.5 * a * math.erfc(-a / 2 ** 0.5) for a in w])
    rel = (2 * (w * w + 1) + 32 + 2) * 2.0 ** -24
    rounding = U[dt] if dt != "f32" else 0.0
    bound = np.abs(want) * (rel + rounding * (1 + rel)) + (TINY[dt] if dt == "f16" else 0.0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), w[bad][:3], got[bad][:3], want[bad][:3])

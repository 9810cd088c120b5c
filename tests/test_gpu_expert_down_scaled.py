"""The experts' down products where they go through memory as fp16 numbers that
share an exponent (bf16, many rows, top_k > 1): magnitudes from the smallest to
the largest, zeros, and rows that hold infinities or NaN."""
import numpy as np
import pytest
import torch

import synth
from tests import test_gpu_expert_ffn as ffn

pytestmark = pytest.mark.gpu


def _run(x, w_up, w_down, idx, weights):
    from paper_2511_19457_amd import abi
    t, k, e = x.shape[0], idx.shape[1], w_up.shape[0]
    dev = torch.device("cuda")
    d = abi.expert_ffn_desc(t, k, e, x.shape[1], w_down.shape[2], x.dtype)
    plan = torch.empty(abi.sparoa_expert_plan_words(t, k, e), dtype=torch.int32, device=dev)
    abi.sparoa_expert_plan(t, k, e, torch.from_numpy(idx).to(dev), plan, torch.empty(
        abi.sparoa_expert_plan_workspace_size(t, k, e), dtype=torch.uint8, device=dev))
    ws = torch.full((abi.sparoa_expert_ffn_workspace_size(d),), 255, dtype=torch.uint8, device=dev)
    y = torch.zeros_like(x, device=dev)
    abi.sparoa_expert_ffn(d, abi.ACT_NONE, x.to(dev), w_up.to(dev), None, w_down.to(dev), None,
                          torch.from_numpy(weights).to(dev), plan, None, y, ws)
    return y


@pytest.mark.parametrize("power", [-120, -60, -14, 0, 17, 60, 118])
@pytest.mark.parametrize("hidden", [128, 131])
def test_magnitudes(power, hidden):
    """Tokens of 2^power and of a thousandth of it, channels a million apart."""
    t, e, k, inner = 300, 4, 2, 64
    x = synth.normal((t, hidden), "bf16", 9960, std=hidden ** -0.5)
    x[::3] *= 2.0 ** -10
    x[5] = 0
    w_up = synth.normal((e, inner, hidden), "bf16", 9961)
    w_down = synth.normal((e, hidden, inner), "bf16", 9962, std=inner ** -0.5)
    w_down = (w_down.float() * 2.0 ** power).to(torch.bfloat16)
    if power > -100:
        w_down[:, 3::8] = (w_down[:, 3::8].float() * 2.0 ** -20).to(torch.bfloat16)
    idx = ffn.choices(t, k, e, "even", 5)
    weights = (np.random.default_rng(6).random((t, k)) + 0.1).astype(np.float32)
    ref, err = ffn.reference(x, w_up, None, w_down, None, idx, weights, None, False, "none", "bf16")
    got = _run(x, w_up, w_down, idx, weights).double().cpu().numpy()
    # a channel far below its neighbours: fp16's last step below the block's largest
    top = np.abs(ref).max(1, keepdims=True)
    bad = ~(np.abs(got - ref) <= err + top * 2.0 ** -20)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:3].tolist())
    assert not got[5].any()


def test_rows_with_infinities_keep_to_themselves():
    t, e, k, hidden, inner = 400, 4, 2, 64, 64
    x = synth.normal((t, hidden), "bf16", 9963)
    w_up = synth.normal((e, inner, hidden), "bf16", 9964, std=0.1)
    w_down = synth.normal((e, hidden, inner), "bf16", 9965, std=0.1)
    idx = ffn.choices(t, k, e, "even", 7)
    weights = np.full((t, k), 0.5, np.float32)
    clean = _run(x, w_up, w_down, idx, weights)
    x[9, 3], x[200, 0], x[399, 63] = float("nan"), float("inf"), float("-inf")
    got = _run(x, w_up, w_down, idx, weights)
    bad = torch.zeros(t, dtype=torch.bool, device="cuda")
    bad[[9, 200, 399]] = True
    assert torch.equal(got[~bad], clean[~bad]) and not torch.isfinite(got[bad]).any()


def test_an_infinite_channel_keeps_to_its_expert():
    """One channel of one expert infinite: that channel of its tokens, finite
    neighbours still within plain fp16 of their values."""
    t, e, k, hidden, inner = 400, 4, 2, 64, 64
    x = synth.normal((t, hidden), "bf16", 9966).abs() + 0.5
    w_up = synth.normal((e, inner, hidden), "bf16", 9967, std=0.1).abs()
    w_down = synth.normal((e, hidden, inner), "bf16", 9968, std=0.1)
    idx = ffn.choices(t, k, e, "even", 8)
    weights = np.full((t, k), 0.5, np.float32)
    ref, err = ffn.reference(x, w_up, None, w_down, None, idx, weights, None, False, "none", "bf16")
    w_down[2, 17] = float("inf")
    got = _run(x, w_up, w_down, idx, weights).double().cpu().numpy()
    mine = (idx == 2).any(1)
    assert np.isposinf(got[mine, 17]).all()
    got[mine, 17], ref[mine, 17] = 0, 0
    assert (np.abs(got - ref) <= err).all()

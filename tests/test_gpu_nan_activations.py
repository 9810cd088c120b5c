"""A NaN passes the activations of the experts' products and of adapted FCs: a row
that holds one gives NaN, whatever kernel serves it."""
import numpy as np
import pytest
import torch

import synth
from tests import test_gpu_expert_ffn as ffn
from tests.test_gpu_expert_precision import call

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "relu6"]


# few rows, rows off 16 bytes, 64 x 64 and 64 x 128 tiles
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("t,e,k,hidden,inner", [(6, 4, 2, 64, 64), (6, 4, 2, 61, 35),
                                                (300, 4, 1, 64, 72), (300, 4, 2, 200, 264),
                                                (900, 2, 2, 61, 520)])
def test_experts(act, dt, t, e, k, hidden, inner):
    x = synth.normal((t, hidden), dt, 9990)
    w_up = synth.normal((e, inner, hidden), dt, 9991, std=hidden ** -0.5)
    w_down = synth.normal((e, hidden, inner), dt, 9992, std=inner ** -0.5)
    idx = ffn.choices(t, k, e, "even", 9)
    weights = np.ones((t, k), np.float32)
    x[t - 1, hidden - 1] = float("nan")
    got = call(x, w_up, w_down, idx, weights, act=act)
    assert np.isnan(got[t - 1]).all() and np.isfinite(got[:t - 1]).all()


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,k,n", [(5, 64, 40), (5, 61, 37), (90, 61, 72), (700, 256, 520),
                                   (2100, 128, 1500)])
def test_adapted(act, dt, m, k, n):
    from paper_2511_19457_amd import abi
    dev = torch.device("cuda")
    x = synth.normal((m, k), dt, 9993)
    w = synth.normal((n, k), dt, 9994, std=k ** -0.5)
    a = synth.normal((3, 8, k), dt, 9995, std=k ** -0.5)
    b = synth.normal((3, n, 8), dt, 9996, std=0.5)
    ids = (np.arange(m) % 3 - 1).astype(np.int32)        # -1, 0, 1; nobody names 2
    x[0, k // 2] = x[m - 1, 0] = float("nan")            # without an adapter, and with one
    b[1, n - 1, 3] = float("nan")                        # the last channel of adapter 1
    d = abi.fc_adapted_desc(m, k, n, 3, 8, x.dtype)
    ws = torch.full((abi.sparoa_fc_adapted_workspace_size(d),), 255, dtype=torch.uint8, device=dev)
    y = torch.zeros(m, n, dtype=x.dtype, device=dev)
    abi.sparoa_fc_adapted(d, act, x.to(dev), w.to(dev), None, a.to(dev), b.to(dev),
                          torch.ones(3, device=dev), torch.from_numpy(ids).to(dev), None, y, ws)
    bad = np.zeros((m, n), bool)
    bad[[0, m - 1]] = True
    bad[ids == 1, n - 1] = True
    assert np.array_equal(torch.isnan(y).cpu().numpy(), bad)

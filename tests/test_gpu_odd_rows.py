"""Experts and adapted FCs whose rows start off 16 bytes, on both sides of the
sizes from which they are copied to aligned rows; tolerances of the aligned
tests."""
import pytest
import torch

import synth
from tests import test_gpu_expert_ffn as ffn
from tests import test_gpu_fc_adapted as fc

pytestmark = pytest.mark.gpu

# tokens, experts, choices, hidden, inner
EXPERTS = [(60, 4, 2, 50, 99), (66, 4, 2, 50, 99), (33, 1, 1, 1, 3), (200, 4, 2, 203, 64),
           (200, 4, 2, 64, 203), (97, 2, 2, 35, 37), (900, 3, 2, 259, 517), (1500, 9, 1, 1021, 70)]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", EXPERTS)
def test_experts(shape, gated, dt):
    i = EXPERTS.index(shape)
    ffn.run(*shape, dt, gated, ("silu", "gelu", "none")[i % 3], bias=i % 2 == 0,
            residual=i % 2 == 1, seed=70 + i)


@pytest.mark.parametrize("kind", ["one", "padded", "empty"])
def test_experts_masked(kind):
    ffn.run(400, 8, 2, 131, 77, "bf16", True, "silu", kind=kind, bias=True, residual=True,
            poison=True, seed=80)
    ffn.run(400, 3, 2, 133, 66, "f32", False, "relu", kind=kind, poison=True, seed=81)


# m, k, n, adapters, rank
ADAPTED = [(64, 33, 47, 5, 3), (65, 33, 47, 5, 3), (130, 1001, 64, 2, 20), (300, 301, 520, 9, 8),
           (1000, 515, 1032, 16, 64), (70, 9, 8, 80, 16), (2100, 1023, 260, 3, 16)]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("kind", ["runs", "mixed", "none"])
@pytest.mark.parametrize("shape", ADAPTED)
def test_adapted(shape, kind, dt):
    i = ADAPTED.index(shape)
    fc.run(*shape, dt, kind=kind, act=i % 3, bias=i % 2 == 0, residual=i % 2 == 1,
           poison=True, seed=50 + i)


def test_a_row_with_nan_keeps_to_itself():
    from paper_2511_19457_amd import abi
    m, k, n = 200, 77, 90
    x = synth.normal((m, k), "bf16", 9950).cuda()
    w = synth.normal((n, k), "bf16", 9951).cuda()
    a, b = synth.normal((2, 8, k), "bf16", 9952).cuda(), synth.normal((2, n, 8), "bf16", 9953).cuda()
    ids = (torch.arange(m, device="cuda") % 3 - 1).int()
    scale = torch.ones(2, device="cuda")
    d = abi.fc_adapted_desc(m, k, n, 2, 8, torch.bfloat16)
    ws = torch.full((abi.sparoa_fc_adapted_workspace_size(d),), 255, dtype=torch.uint8,
                    device="cuda")
    clean, y = torch.empty(m, n, dtype=x.dtype, device="cuda"), None
    abi.sparoa_fc_adapted(d, abi.ACT_NONE, x, w, None, a, b, scale, ids, None, clean, ws)
    x[50, k - 1], x[7, 0] = float("nan"), float("inf")
    y = torch.empty_like(clean)
    abi.sparoa_fc_adapted(d, abi.ACT_NONE, x, w, None, a, b, scale, ids, None, y, ws)
    bad = torch.zeros(m, dtype=torch.bool, device="cuda")
    bad[[7, 50]] = True
    assert torch.equal(y[~bad], clean[~bad]) and not torch.isfinite(y[bad]).any()

"""Experts' products and adapted FCs in their largest tiles: 128 x 256 for the
16-bit types (and 64 x 128 of adapted FCs), 64 x 128 for fp32; which tile a shape
runs is asserted by test_row_tile_launches.py.  More tiles than work-groups on the
chip, segments of every length, widths off a vector and K of a dozen and more
chunks with a rest.  References and tolerances of the small shapes' tests."""
import pytest

from tests import test_gpu_expert_ffn as ffn
from tests import test_gpu_fc_adapted as fc

pytestmark = pytest.mark.gpu

# tokens, experts, choices, hidden, inner, gated, how the choices lie
EXPERTS = [(2100, 16, 4, 1304, 696, True, "even"), (2100, 16, 4, 1300, 700, True, "one"),
           (2100, 16, 4, 1304, 1304, False, "one"), (2100, 16, 4, 1300, 1300, False, "padded"),
           (8400, 16, 1, 1304, 696, True, "padded")]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", EXPERTS)
def test_experts(shape, dt):
    i = EXPERTS.index(shape)
    ffn.run(*shape[:5], dt, shape[5], ("silu", "gelu", "relu", "none", "relu6")[i], kind=shape[6],
            bias=i % 2 == 1, residual=i % 2 == 0, poison=i == 3, seed=90 + i)


# m, k, n, adapters, rank, the 16-bit types' tile
ADAPTED = [(1500, 1000, 1500, 5, 20, "64x128"), (1500, 968, 1501, 9, 16, "64x128"),
           (2000, 808, 2801, 6, 40, "128x256"), (4100, 840, 2500, 12, 20, "128x256"),
           (4100, 1000, 2501, 7, 16, "128x256")]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", ADAPTED)
@pytest.mark.parametrize("kind", ["runs", "mixed"])
def test_adapted(shape, kind, dt):
    i = ADAPTED.index(shape)
    fc.run(*shape[:5], dt, kind=kind, act=i % 3, bias=True, residual=i % 2 == 0, seed=60 + i)

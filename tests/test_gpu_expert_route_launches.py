"""Routing and plan around the sizes where the launches change: one work-group
or two launches, work-groups of 4 or 16 waves."""
import numpy as np
import pytest

from tests.test_gpu_expert_route import check, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,e", [(8, 257), (9, 257), (16, 65), (17, 65), (32, 64), (33, 64),
                                 (256, 12), (257, 12), (1024, 66), (1025, 66), (1000, 300)])
@pytest.mark.parametrize("score", [0, 1])
def test_sizes(t, e, score):
    check(logits(t, e, "bf16", t + e), 5, score=score, renorm=True)
    mask = (np.random.default_rng(t).random(t) < 0.7).astype(np.uint8)
    check(logits(t, e, "f32", t), 2, score=score, mask=mask, scale=2.5)

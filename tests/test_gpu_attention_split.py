"""Batches whose work lies at a step of the split's ranges: the kernels that find the split
each for themselves find the same one (an output of another split would miss ranges or
take some twice)."""
import pytest

from tests.test_gpu_paged_attention import Batch, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [1, 2])
@pytest.mark.parametrize("more", [-65, -1, 0, 1, 2, 64])
def test_single_rows(more, steps, dt):
    """8 kv heads, 1024 items wanted: a range is a tile of 64 keys longer from 8192 keys of
    all requests on, and again from 16384."""
    total = 8192 * steps + more
    for shares in ((1.0,), (0.5, 0.5), (0.31, 0.0, 0.09, 0.6), tuple([1 / 33] * 33)):
        keys = [max(1, int(total * s)) for s in shares]
        keys[-1] = max(1, keys[-1] + total - sum(keys))
        compare(Batch([1] * len(keys), keys, 8, 8, 8, 64, dt, seed=steps))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("more", [-1, 0, 1])
def test_rows_of_several_tiles(more, dt):
    for rows, keys in (([130, 40, 260], [1280 + more, 640, 2560]), ([200] * 3, [2048 + more, 200, 4096]),
                       ([64, 64 + more, 300], [64, 4096, 5120 + more])):
        compare(Batch(rows, keys, 4, 2, 40, 16, dt, seed=5))

"""sparoa_block_norm of rows that are no multiple of a 16-byte vector, around
the lengths where its kernel changes, with the tolerance of the other norm
tests."""
import pytest

from tests.test_gpu_block_norm import _run

pytestmark = pytest.mark.gpu

COLS = [255, 257, 1001, 1023, 1025, 3001, 4095, 4097, 6811, 8190, 16383, 16385]


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cols", COLS)
def test_row_lengths(dt, cols):
    i = COLS.index(cols)
    _run(1 + i % 6, cols, dt, post=i % 3, pre=1 + (i + 1) % 2, gate_rows=1 + i % 3, c=0.5, seed=i)
    _run(3, cols, dt, post=2, pre=2, mean=100.0, seed=70)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("post,pre", [(0, 0), (0, 1), (0, 2), (1, 0), (1, 1), (2, 2)])
@pytest.mark.parametrize("cols", [77, 513, 1031, 5001])
def test_operands(dt, post, pre, cols):
    _run(9, cols, dt, post, pre, seed=71)
    _run(9, cols, dt, post, pre, gate_rows=4, affine=False, c=-2.0, seed=72)
    _run(9, cols, dt, post, pre, has_r=False, seed=73)
    if pre:
        _run(9, cols, dt, post, pre, has_y=False, write_r=False, seed=74)
    _run(9, cols, dt, post, max(pre, 1), gate_rows=9, in_place=True, seed=75)


@pytest.mark.parametrize("cols", [33, 515, 1029, 4099])
def test_more_rows_than_work_groups(cols):
    _run(5000, cols, "bf16", post=1, pre=1, gate_rows=5000, seed=76)

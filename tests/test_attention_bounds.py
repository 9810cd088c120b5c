"""Sizes of the attention calls next to their bounds, on the CPU (launches are recorded,
not run): which are served, by launches that cover every item, and which refused."""
import pytest

from tests.test_attention_launches import desc, launches  # noqa: F401

ONE = dict(max_queries=1, table_pages=1, max_keys=16)
SERVED = [
    # (what the descriptor has, row tiles that its batches may have)
    (dict(tokens=1 << 20, requests=1 << 20, heads=8, kv_heads=8, **ONE), 1 << 20),
    (dict(tokens=66000, requests=66000, heads=128, kv_heads=128, **ONE), 66000),
    (dict(tokens=1 << 24, requests=1 << 24, heads=4, kv_heads=4, **ONE), 1 << 24),
    (dict(tokens=(1 << 27) - 2048, requests=1, max_queries=(1 << 27) - 2048), ((1 << 27) - 2048) // 32),
    (dict(tokens=1 << 26, heads=16, kv_heads=16, requests=1 << 16, max_queries=1 << 26),
     (1 << 19) + (1 << 16)),
    (dict(tokens=8, requests=1 << 24, table_pages=100, max_keys=1600), 8),
    (dict(heads=2048, kv_heads=2048), 2), (dict(heads=1 << 20, kv_heads=1, tokens=64), 1 << 17),
    (dict(heads=1 << 20, kv_heads=1 << 20, tokens=64, requests=64, **ONE), 64),
    (dict(max_keys=(1 << 31) - 2048, table_pages=1 << 27, requests=1), 1)]


@pytest.mark.parametrize("kind", ["attend", "tree"])
def test_served(launches, kind):
    calls = [(desc(**d), tiles) for d, tiles in SERVED
             if kind == "attend" or d.get("max_queries", 8) <= 256]
    for (d, tiles), (status, got) in zip(calls, launches([[kind, d] for d, _ in calls])):
        assert status == 0, d
        grids = [x for name, x, y, z in got if "attention_kernel" in name]
        assert all(0 < x * 256 < 1 << 32 and x % d["kv_heads"] == 0 for x in grids), (d, grids)
        assert sum(grids) >= tiles * d["kv_heads"], (d, grids)
        # (no request without a token has work-groups: they would outnumber the others)
        assert sum(grids) <= (2 * tiles + 2 * 1024) * d["kv_heads"] + 2 * 1024, (d, grids)

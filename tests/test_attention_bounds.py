"""Sizes of the attention calls next to their bounds, on the CPU (launches are recorded,
not run): which are served, by launches that cover every item, and which refused."""
import os
import subprocess

import pytest

from tests.test_attention_launches import HERE, desc, launches  # noqa: F401

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


SIZES = ("tokens", "requests", "heads", "pages", "page_size", "table_pages", "max_keys")
FAR = ((1 << 63) - 1, (1 << 63) - 1024, (1 << 62) + 2, 1 << 32)


@pytest.mark.parametrize("kind", ["attend", "tree", "append", "keep"])
def test_sizes_at_the_end_of_64_bits(launches, kind):
    """No sum or product of sizes wraps round into the bounds."""
    calls = [[kind, desc(**{n: v - v % 2 if n == "heads" else v})] for n in SIZES for v in FAR]
    for (_, d), (status, got) in zip(calls, launches(calls)):
        assert status in (1, 2) and not got, d


PROGRAM = r"""
#include <cstdio>
#include "cache.h"
namespace sparoa {
sparoa_status fail(sparoa_status s, const std::string &) { return s; }
void clear_error() {}
size_t attention_workspace(const sparoa_kv_desc &) { return 0; }
sparoa_status launch_kv_append(const AppendArgs &, sparoa_dtype, hipStream_t) { return SPAROA_OK; }
sparoa_status launch_kv_keep(const KeepArgs &, int64_t, sparoa_dtype, hipStream_t) { return SPAROA_OK; }
sparoa_status launch_attention(AttnArgs, const sparoa_kv_desc &, void *, hipStream_t) {
  return SPAROA_OK;
}
}
int main() {
  size_t bytes;
  const int64_t far[] = {INT64_MAX, INT64_MAX - 1023, ((int64_t)1 << 62) + 2, (int64_t)1 << 32};
  for (int64_t v : far)
    for (int i = 0; i < 10; ++i) {
      int64_t s[10] = {8, 2, 8, 2, 64, 20, 16, 10, 8, 160};
      s[i] = v;
      const sparoa_kv_desc d{s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7], s[8], s[9], SPAROA_BF16};
      if (sparoa_attention_workspace_size(&d, &bytes) != SPAROA_OK) continue;
      if (i != 8) return printf("size %d of %lld is taken\n", i, (long long)v), 1;
    }
  return 0;
}
"""


def test_no_check_overflows(tmp_path):
    """The argument checks by themselves, in a build that stops where a signed sum passes its
    type."""
    (tmp_path / "checks.cpp").write_text(PROGRAM)
    root = os.path.dirname(HERE)
    csrc = os.path.join(root, "paper_2511_19457_amd", "csrc")
    exe = str(tmp_path / "checks")
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-O1",
                    "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all",
                    "-I", "/opt/rocm/include", "-I", os.path.join(root, "include"), "-I", csrc,
                    os.path.join(csrc, "cache_abi.cpp"), str(tmp_path / "checks.cpp"), "-o", exe],
                   check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr

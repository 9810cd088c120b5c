"""Launches of the attention calls, on the CPU: recorded instead of run
(launch_recorder.c), in a process of its own.  No launch is larger than the runtime
takes (2^32 threads a dimension) whatever the descriptor's bounds; batches above 64
requests are planned in front; a cache that no range is cut of is not joined."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

PROGRAM = r"""
import ctypes, json, sys
import torch                     # (its own libraries keep the real runtime)
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
rec.recorded_name.restype = ctypes.c_char_p
from paper_2511_19457_amd import abi
out, p = [], 1 << 20
for kind, desc in json.loads(sys.argv[2]):
    d = abi.KvDesc(**desc)
    o = abi.attention_opts(0.1)
    rec.forget_launches()
    if kind == "append":
        st = abi._L.sparoa_kv_append(ctypes.byref(d), 8, 0, p, d.heads * d.head_dim, p,
                                     d.kv_heads * d.head_dim, p, d.kv_heads * d.head_dim, p, None,
                                     p, p, p, 2 * p, p, p, None)
    elif kind == "keep":
        st = abi._L.sparoa_kv_keep(ctypes.byref(d), 100, p, p, p, p, 8, p, p, p, None)
    elif kind == "tree":
        st = abi._L.sparoa_tree_attention(ctypes.byref(d), ctypes.byref(o), p, p, p, p, p, p, p,
                                          None, None, p, p, 1 << 60, None)
    else:
        st = abi._L.sparoa_paged_attention(ctypes.byref(d), ctypes.byref(o), p, p, p, p, p, p,
                                           None, None, None, p, p, 1 << 60, None)
    got = []
    for i in range(rec.recorded_launches()):
        grid = (ctypes.c_uint * 3)()
        rec.recorded_grid(i, grid)
        got.append([rec.recorded_name(i).decode(), *grid])
    out.append([st, got])
print("LAUNCHES" + json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("recorder") / "launch_recorder.so")
    subprocess.run(["gcc", "-std=c11", "-O1", "-fPIC", "-shared", "-o", so,
                    os.path.join(HERE, "launch_recorder.c")], check=True)

    def run(calls):
        r = subprocess.run([sys.executable, "-c", PROGRAM, so, json.dumps(calls)],
                           cwd=os.path.dirname(HERE), capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout.split("LAUNCHES")[1])
    return run


def desc(**kw):
    d = dict(tokens=8, requests=2, heads=8, kv_heads=2, head_dim=64, pages=20, page_size=16,
             table_pages=10, max_queries=8, max_keys=160, dtype=2)
    d.update(kw)
    return d


LARGE = [dict(tokens=(1 << 27) - 2048, max_queries=1 << 20), dict(tokens=1 << 20, requests=1 << 20),
         dict(tokens=1 << 26, heads=16, kv_heads=16, requests=1 << 16, max_queries=1 << 26),
         dict(requests=1 << 24, table_pages=100, max_keys=1600), dict(heads=2048, kv_heads=2048),
         dict(heads=1 << 20, kv_heads=1, tokens=64),
         dict(max_keys=(1 << 31) - 2048, table_pages=1 << 27, requests=1)]


@pytest.mark.parametrize("kind", ["attend", "tree", "append", "keep"])
def test_grids(launches, kind):
    wide = dict(max_queries=256) if kind == "tree" else {}
    for d, (status, got) in zip(LARGE, launches([[kind, desc(**{**d, **wide})] for d in LARGE])):
        assert status in (0, 2), d          # (too many rows are refused)
        assert bool(got) == (status == 0), d
        for name, x, y, z in got:
            threads = 1024 if "plan" in name else 256
            assert 0 < x * threads < 1 << 32 and 0 < y < 65536 and 0 < z < 65536, (d, name, x, y, z)


def names(got):
    return [next(k for k in ("plan_kernel", "attention_kernel", "join_kernel") if k in g[0])
            for g in got]


def test_kernels(launches):
    got = launches([["attend", desc(requests=64)], ["attend", desc(requests=65)],
                    ["tree", desc(requests=65)], ["attend", desc(max_keys=64)],
                    ["attend", desc(requests=65, max_keys=64)], ["attend", desc(max_keys=65)]])
    assert [g[0] for g in got] == [0] * 6
    assert [names(g[1]) for g in got] == [
        ["attention_kernel", "join_kernel"], ["plan_kernel", "attention_kernel", "join_kernel"],
        ["plan_kernel", "attention_kernel", "join_kernel"], ["attention_kernel"],
        ["plan_kernel", "attention_kernel"], ["attention_kernel", "join_kernel"]]

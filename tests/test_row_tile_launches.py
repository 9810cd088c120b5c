"""Kernels and tiles of the experts' products and adapted FCs, on the CPU: the
library's launches are recorded instead of run (launch_recorder.c), in a process of
its own.  The shapes of test_gpu_row_tiles.py run the tiles that they are there
for, and no launch is larger than the runtime takes (2^32 threads a dimension)."""
import json
import os
import re
import subprocess
import sys

import pytest

from tests.test_gpu_row_tiles import ADAPTED, EXPERTS

HERE = os.path.dirname(os.path.abspath(__file__))
CODE = {"f32": 0, "f16": 1, "bf16": 2}

PROGRAM = r"""
import ctypes, json, sys
import torch                     # (its own libraries keep the real runtime)
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
rec.recorded_name.restype = ctypes.c_char_p
from paper_2511_19457_amd import abi
out, p = [], 1 << 20
for kind, dt, *v in json.loads(sys.argv[2]):
    grid, got = (ctypes.c_uint * 3)(), []
    rec.forget_launches()
    if kind == "experts":
        t, e, k, h, i, gated = v
        d = abi.expert_ffn_desc(t, k, e, h, i, dt, gated=bool(gated))
        st = abi._L.sparoa_expert_ffn(ctypes.byref(d), 0, p, p, None, p, None, p, p, None, p, p,
                                      1 << 60, None)
    else:
        d = abi.fc_adapted_desc(*v, dt)
        st = abi._L.sparoa_fc_adapted(ctypes.byref(d), 0, p, p, None, p, p, p, p, None, p, p,
                                      1 << 60, None)
    for i in range(rec.recorded_launches()):
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


def tiles(got):
    """{mode: tile} of the products launched: rows x weight rows, or "split"."""
    out = {}
    for name, *_ in got:
        m = re.search(r"rows_(tile|split|stream)_kernelILi\dELNS_8RowsModeE(\d)E((?:Li\d+E)+)", name)
        if not m:
            continue
        v = [int(i) for i in re.findall(r"Li(\d+)E", m.group(3))]
        out[int(m.group(2))] = "%dx%d" % (16 * v[0] * v[2], 16 * v[1] * v[3]) \
            if m.group(1) == "tile" else m.group(1)
    return out


UP, GATED, SCALED, DOWN, FC = range(5)


def test_shapes_run_the_tiles_they_are_for(launches):
    cases = [(s, dt) for s in EXPERTS for dt in CODE]
    for (s, dt), (st, got) in zip(cases, launches(
            [["experts", CODE[dt], *s[:6]] for s, dt in cases])):
        down = SCALED if dt == "bf16" and s[2] > 1 else DOWN
        want = "64x128" if dt == "f32" else "128x256"
        assert st == 0 and tiles(got) == {GATED if s[5] else UP: want, down: want}, (s, dt, got)
    cases = [(s, dt) for s in ADAPTED for dt in CODE]
    for (s, dt), (st, got) in zip(cases, launches(
            [["adapted", CODE[dt], *s[:5]] for s, dt in cases])):
        want = "64x128" if dt == "f32" else s[5]
        assert st == 0 and tiles(got)[FC] == want, (s, dt, got)


def threads(name):
    m = re.search(r"rows_split_kernelILi\dELNS_8RowsModeE\dELi\d+ELi\d+ELi(\d+)E", name)
    if m:
        return 64 * int(m.group(1))
    m = re.search(r"rows_tile_kernelILi\dELNS_8RowsModeE\dELi(\d+)ELi(\d+)E", name)
    if m:
        return 64 * int(m.group(1)) * int(m.group(2))
    return 512 if "rows_stream" in name else 256


# m, k, n, adapters, rank: very many short rows, aligned and padded
HUGE = [(1 << 26, 8, 8, 2, 16), (1 << 27, 8, 8, 2, 16), ((1 << 27) + 5, 8, 8, 2, 16),
        (1 << 28, 64, 64, 2, 64), (1 << 25, 8, 8, 2, 512), (1 << 29, 8, 8, 2, 8),
        ((1 << 24) * 32, 57, 8, 2, 8), ((1 << 24) * 32 - 3, 57, 8, 2, 8), (1 << 29, 8, 8, 3, 512)]


def test_launches_of_very_many_rows_fit(launches):
    for dt in (0, 2):
        for s, (st, got) in zip(HUGE, launches([["adapted", dt, *s] for s in HUGE])):
            assert st == 0 and got, s
            for name, x, y, z in got:
                assert x * threads(name) < 1 << 32 and y < 1 << 16, (s, dt, name, x, y)

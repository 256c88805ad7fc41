"""Which kernels the attention and cache calls launch (CPU: a stand-in for the runtime writes the launches down): the sizes of the
GPU tests reach every kernel that is compiled, each launch asks for the LDS that it may, and none keeps registers in memory."""
import json
import os
import re
import subprocess
import sys

import pytest

from tests.test_op_forms import OBJDUMP, compiled

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
READELF = "/opt/rocm/llvm/bin/llvm-readelf"
SOURCES = ["k_kv.hip", "k_kv_attend.hip", "k_kv_attend_rows.hip", "k_attend.hip", "k_attend_rows.hip", "k_attend_join.hip"]
DIMS = (8, 32, 40, 64, 72, 80, 96, 120, 128, 136, 192, 200, 256)

_CHILD = """
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
shim.launch_log_take.restype = ctypes.c_char_p
from paper_2607_12287_amd import incvit
incvit.lib()
def take():
    return [line.split() for line in shim.launch_log_take().decode().splitlines()]
out = []
R = incvit.incvit_rows
for c in json.load(sys.stdin):
    take()
    d, hk, dt = c["d"], c["hk"], c["dtype"]
    kv = incvit.incvit_kv(1 << 20, c.get("block", 16), hk, d)
    A, B, C, D, E, F = (1 << k for k in range(40, 46))
    if c["op"] == "write":
        st = incvit.incvit_kv_write(kv, dt, c["rows"], A, hk * d, d, B, hk * d, d, C, 1, D)
    elif c["op"] == "read":
        st = incvit.incvit_kv_read(kv, D, dt, c["rows"], C, 0, A, hk * d, d, B, hk * d, d)
    else:
        hq, n = c["hq"], c["n"]
        a = incvit.incvit_attention(dt, hq, hk, d, 1, c.get("window", 0), 0, 0, 1.0)
        q, o, kr = R(A, hq * d, d), R(B, hq * d, d), R(C, hk * d, d)
        starts = F if c.get("ragged") else 0
        if c["op"] == "cached":
            st = incvit.incvit_kv_attend(a, kv, D, n, c["rows"], starts, E, 1 << 16, c["keys"] // 16 + 1, F, c["keys"], q, o, 1 << 46)
        else:
            st = incvit.incvit_attend(a, n, c["rows"], starts, n * c["keys"], starts, c["keys"], q, kr, kr, o, 1 << 46)
    assert st == 0, (c, st, incvit.incvit_last_error())
    out.append(take())
print("LAUNCHES " + json.dumps(out))
"""


def launches(calls, tmp_path):
    """Per call its launches [(kernel, grid x, y, z, threads, LDS bytes)]."""
    shim = str(tmp_path / "launch_log.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "launch_log.cpp")])
    res = subprocess.run([sys.executable, "-c", _CHILD, shim], input=json.dumps(calls), cwd=ROOT, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    out = json.loads(next(line for line in res.stdout.splitlines() if line.startswith("LAUNCHES "))[9:])
    flat = sorted({e[0] for c in out for e in c})
    names = dict(zip(flat, subprocess.run(["c++filt"], input="\n".join(flat), capture_output=True, text=True, check=True).stdout.splitlines()))

    def short(n):
        n = names[n].replace("(anonymous namespace)::", "").replace("incvit::", "").replace("void ", "").split("(")[0]
        return re.sub(r"\s+", "", n).replace("unsignedshort", "bf16")

    return [[(short(e[0]), *(int(v) for v in e[1:])) for e in c] for c in out]


def gpu_test_calls():
    """The calls of test_gpu_kv and test_gpu_attend, as far as kernels go."""
    for dt in (0, 1):
        for d in DIMS:
            for block in (16, 32, 64, 128):
                yield dict(op="write", d=d, hk=2, dtype=dt, rows=2 * block + block // 2 + 3, block=block)
            yield dict(op="read", d=d, hk=2, dtype=dt, rows=80)
            yield dict(op="plain", d=d, hk=1, hq=4, dtype=1, n=3, rows=8462, keys=8192, ragged=1)
            for op in ("cached", "plain"):
                for nq in (1, 5, 9, 70):
                    yield dict(op=op, d=d, hk=1, hq=4, dtype=dt, n=2, rows=2 * nq, keys=99)
                for nq in (1, 30, 150):  # keys shared by workgroups
                    yield dict(op=op, d=d, hk=2, hq=8, dtype=dt, n=2, rows=2 * nq, keys=3000)


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not installed")
def test_every_kernel_is_launched_by_the_gpu_tests(tmp_path):
    got = launches(list(gpu_test_calls()), tmp_path)
    reached = {e[0] for c in got for e in c}
    built = set()
    for source in SOURCES:
        built |= compiled(tmp_path, source)
        for f in os.listdir(tmp_path):
            if f.startswith("k_"):
                os.remove(tmp_path / f)
    assert sorted(built - reached) == []
    for c in got:
        for _, x, y, z, threads, lds in c:
            assert x * y * z * threads < 2 ** 32 and lds <= 160 * 1024


@pytest.mark.skipif(not os.path.exists(READELF), reason="llvm-readelf not installed")
@pytest.mark.parametrize("source", SOURCES)
def test_no_kernel_keeps_registers_in_memory(source, tmp_path):
    compiled(tmp_path, source)
    code = [f for f in os.listdir(tmp_path) if f.endswith("gfx950")]
    notes = subprocess.check_output([READELF, "--notes", code[0]], cwd=tmp_path, text=True)
    spills = re.findall(r"\.vgpr_spill_count:\s+(\d+)", notes)
    assert spills and set(spills) == {"0"}, spills


def test_splits(tmp_path):
    """One launch for few keys or many rows; the join behind it where workgroups share keys."""
    def kernels(**c):
        return [e[0].split("<")[0] for e in launches([dict(dict(d=128, hk=4, hq=16, dtype=1, n=1, rows=1, keys=1024), **c)], tmp_path)[0]]

    assert kernels(op="cached") == ["kv_attend_kernel"] and kernels(op="plain") == ["attend_kernel"]
    assert kernels(op="cached", keys=1100) == ["kv_attend_kernel", "attend_join_kernel"]
    assert kernels(op="plain", keys=9000, n=30, rows=30) == ["attend_kernel", "attend_join_kernel"]
    assert kernels(op="cached", keys=500, rows=64) == ["kv_attend_kernel"] and kernels(op="plain", keys=500, rows=32) == ["attend_kernel"]
    assert kernels(op="cached", keys=500, n=16, rows=320) == ["kv_attend_rows_kernel"]
    assert kernels(op="plain", keys=500, n=16, rows=80) == ["attend_rows_kernel"]
    assert kernels(op="plain", keys=8192, rows=8192) == ["attend_rows_kernel"]
    assert kernels(op="cached", keys=8192, rows=512) == ["kv_attend_rows_kernel", "attend_join_rows_kernel"]
    assert kernels(op="cached", keys=8192, rows=8192, ragged=1) == ["kv_attend_rows_kernel"]
    assert kernels(op="cached", keys=10 ** 6, window=700) == ["kv_attend_kernel"]

"""Calls of the cache and attention operators that are accepted at the edge of their ranges (CPU: a stand-in for the runtime writes
the launches down)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CHILD = """
import ctypes, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
shim.launch_log_take.restype = ctypes.c_char_p
from paper_2607_12287_amd import incvit
incvit.lib()
A, B, C, D, E = (1 << k for k in range(40, 45))
R = incvit.incvit_rows
a, kv = incvit.incvit_attention(1, 8, 4, 64, 1, 0, 0, 0, 0.125), incvit.incvit_kv(100, 16, 4, 64)
def cached(table, width):
    shim.launch_log_take()
    st = incvit.incvit_kv_attend(a, kv, D, 2, 6, 0, table, 50, width, C, 0, R(A, 512, 64), R(E, 512, 64), 0)
    return st, len(shim.launch_log_take().splitlines())
print("GOT", cached(B, 50), cached(0, 0), cached(B, 0), cached(0, 1))
"""


def test_tables_without_columns(tmp_path):
    shim = str(tmp_path / "launch_log.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "launch_log.cpp")])
    res = subprocess.run([sys.executable, "-c", _CHILD, shim], cwd=ROOT, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    from paper_2607_12287_amd import incvit
    ok, arg = (incvit.INCVIT_OK, 1), (incvit.INCVIT_ERR_ARG, 0)
    assert [x for x in res.stdout.splitlines() if x.startswith("GOT")] == [f"GOT {ok} {ok} {ok} {arg}"]

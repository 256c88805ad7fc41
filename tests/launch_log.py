"""Which kernels a call launches, without a GPU: a child process loads the library behind a stand-in for the HIP runtime's
registration and launch functions (launch_log.cpp), makes the calls with addresses that nothing reads, and prints what
would have been launched."""
from __future__ import annotations

import json
import os
import re
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CHILD = """
import ctypes, json, sys
shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
shim.launch_log_take.restype = shim.launch_log_kernels.restype = ctypes.c_char_p
from paper_2607_12287_amd import incvit, synth
incvit.lib()
def take():
    return [line.split() for line in shim.launch_log_take().decode().splitlines()]
calls = json.load(sys.stdin)
out = []
for kind, kw in calls:
    take()
    if kind == "kernels":
        out.append([[n] for n in shim.launch_log_kernels().decode().splitlines()])
        continue
    if kind == "linear":
        f = incvit.incvit_qlinear_multiply if kw.pop("two", 0) else None
        dt, m, K, N = kw["dtype"], kw["rows"], kw["K"], kw["N"]
        x, w, o, q, r = 1 << 40, 1 << 41, (1 << 42) + kw.get("off", 0), 1 << 43, (1 << 44 if kw.get("residual") else 0)
        st = incvit.incvit_qlinear(dt, m, K, N, x, K, w, 0, r, N, o, kw.get("out_stride", N), q)
    elif kind == "quantize":
        K, ln = kw["K"], kw.get("ln", False)
        st = incvit.incvit_qlinear_quantize_rows(kw["dtype"], kw["rows"], K, 1 << 40, kw.get("stride", K), (1 << 41) * ln,
                                                 (1 << 42) * ln, 1e-6, 1 << 43)
    elif kind == "qk":
        dt, m, hq, hk, d, rot = (kw[k] for k in ("dtype", "rows", "hq", "hk", "d", "rot"))
        c = incvit.incvit_qk(dt, d, rot, 0, 1, 1e-6)
        def heads(at, n):
            return incvit.incvit_heads(at + kw.get("off", 0), at + (1 << 36), None, None, n * d, d, n * d, d, n)
        st = incvit.incvit_qk_norm_rope(c, m, heads(1 << 40, hq), heads(1 << 41, hk), 1 << 42, m, 0, 0, 0)
    else:
        m, B = synth.ModelShape(**kw["shape"]), kw["B"]
        st, h = incvit.incvit_create(incvit.make_config(m, B, mlp=kw.get("mlp", "reuse")), 1 << 45)
        assert st == 0, (kw, incvit.incvit_last_error())
        cb = (incvit.incvit_cache_bytes(h) + 255) // 256 * 256
        caches = [(1 << 46) + v * cb for v in range(B)]
        if kind == "full":
            st = incvit.incvit_full_encode(h, B, 1 << 40, caches, 1 << 41)
        else:
            st = incvit.incvit_step(h, B, 1 << 40, caches, kw["tau"], kw["caps"], 1 << 42, 1 << 43, 0, 1 << 41)
        assert st == 0, incvit.incvit_last_error(h)
    assert st == 0, (kind, kw, st, incvit.incvit_last_error())
    out.append(take())
print("LAUNCHES " + json.dumps(out))
"""


def launches(calls, tmp_path):
    """Per call its launches [(kernel, grid x, y, z, threads, LDS bytes)], kernel as name<template arguments>."""
    shim = os.path.join(str(tmp_path), "launch_log.so")
    if not os.path.exists(shim):
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

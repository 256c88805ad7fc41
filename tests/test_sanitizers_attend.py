"""The host side of the cache's and attention's entry points (argument checks, sizes,
the split of the work) under AddressSanitizer and UndefinedBehaviorSanitizer
(CPU): their refusals' tests run against a build whose host pass is instrumented,
in a child process; no kernel runs."""
import glob
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"
RUNTIME = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
INSTRUMENTED = ["incvit_attend.hip"]

pytestmark = pytest.mark.slow


@pytest.mark.skipif(not RUNTIME or not os.path.exists(HIPCC), reason="clang sanitizer runtime not installed")
def test_attention_checks_are_clean_under_asan_and_ubsan(tmp_path):
    from paper_2607_12287_amd import build as hip_build

    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-shared-libsan", "-g", "-O1"]
    host_san = [f for flag in san for f in ("-Xarch_host", flag)]
    objs = hip_build.objects([s for s in hip_build.SOURCES if s not in INSTRUMENTED])
    for s in INSTRUMENTED:
        objs.append(str(tmp_path / (s + ".o")))
        subprocess.check_call([HIPCC, *hip_build.COMMON, *host_san, "-c", os.path.join(hip_build.CSRC, s), "-o", objs[-1]])
    lib = str(tmp_path / "libincvit_san.so")
    link = [f for flag in ("-shared-libsan", san[0]) for f in ("-Xarch_host", flag)]
    subprocess.check_call([HIPCC, "--offload-arch=" + hip_build.ARCH, "-shared", "-fPIC", *link, *objs, "-o", lib])
    env = dict(os.environ, LD_PRELOAD=RUNTIME[0], INCVIT_LIB=lib,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "not gpu and not slow", "-p", "no:cacheprovider",
                          "tests/test_attend_refusals.py"], cwd=ROOT, env=env, capture_output=True, text=True)
    out = res.stdout[-4000:] + res.stderr[-4000:]
    assert res.returncode == 0, out
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out

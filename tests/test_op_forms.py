"""Which kernels the operators' calls launch (CPU: a stand-in for the runtime writes the launches down): the sizes of the GPU
tests take the forms that those tests are about, and every kernel that is compiled for the operators is launched by some call."""
import os
import re
import shutil
import subprocess

import pytest

from tests import test_gpu_options_large as large
from tests import test_gpu_q8_forms as q8
from tests import test_gpu_qk_forms as qk
from tests.launch_log import launches

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
EPI = {("bf16", False): 6, ("f32", False): 7, ("bf16", True): 10, ("f32", True): 11}
ANY = {"bf16": 8, "f32": 9}


def dt(name):
    return 1 if name == "bf16" else 0


def linear(dtype, rows, K, N, residual=False):
    return "linear", dict(dtype=dt(dtype), rows=rows, K=K, N=N, residual=residual)


def full(m, B, **kw):
    return "full", dict(shape=m.__dict__, B=B, **kw)


def only(entries, prefix):
    return [e[0] for e in entries if e[0].startswith(prefix)]


def test_products_take_the_forms_of_their_tests(tmp_path):
    calls, want = [], []
    for forms, wide in ((q8.FORMS, True), (q8.FORMS_ANY, False)):
        for rows, K, N, form in forms:
            for dtype in ("bf16", "f32"):
                for residual in (False, True):
                    kernel, args = form.split()
                    calls.append(linear(dtype, rows, K, N, residual))
                    want.append(f"{kernel}_kernel<{EPI[dtype, residual] if wide else ANY[dtype]},{args}>")
    for call, got, w in zip(calls, launches(calls, tmp_path), want):
        assert got[-1][0] == w, call
    # every form of every epilogue is among them
    reached = {w for w in want if "gemm" in w}
    tiles = {f.split()[1] for *_, f in q8.FORMS if f.startswith("gemm_tiled")}
    few = {f.split()[1] for *_, f in q8.FORMS if f.startswith("q_gemm")}
    assert len(tiles) == 7 and len(few) == 6 and len(reached) == 4 * 13 + 2 * 12


def test_head_norms_take_the_instances_of_their_tests(tmp_path):
    calls = [("qk", dict(dtype=dt(t), rows=rows, hq=hq, hk=hk, d=d, rot=rot)) for t, rows, hq, hk, d, rot, _ in qk.CASES]
    for case, got in zip(qk.CASES, launches(calls, tmp_path)):
        assert [e[0] for e in got] == [f"qk_kernel<{case[-1]}>"], case
    assert len({c[-1] for c in qk.CASES}) == 9 + 6


def test_large_encodes_take_the_kernels_of_their_tests(tmp_path):
    calls = []
    for _, m, B, *_ in large.CASES:
        calls += [full(m, B), ("step", dict(shape=m.__dict__, B=B, tau=float("inf"), caps=[m.n_tokens - 3] * B)), full(m, 1)]
    got = launches(calls, tmp_path)
    for i, (name, m, B, _, down, heads) in enumerate(large.CASES):
        whole, step, one = got[3 * i:3 * i + 3]
        epi = 12 if m.dtype == "bf16" else 13
        assert set(only(whole, "qk_layer")) == {f"qk_layer_kernel<{heads}>"}, name
        for entries in (whole, step):
            assert not down or f"gemm_tiled_kernel<{epi},{down}>" in only(entries, "gemm_tiled"), name
        assert B == 1 or any(k.startswith(f"q_gemm_kernel<{epi},") for k in only(one, "q_gemm")), name


def compiled(tmp_path, source):
    """The kernels in a source's device code."""
    from paper_2607_12287_amd import build as hip_build

    obj = shutil.copy(hip_build.objects([source])[0], tmp_path)
    subprocess.check_call([OBJDUMP, "--offloading", os.path.basename(obj)], cwd=tmp_path, stdout=subprocess.DEVNULL)
    code = [f for f in os.listdir(tmp_path) if f.startswith(os.path.basename(obj)) and f.endswith(hip_build.ARCH)]
    assert len(code) == 1, code
    out = subprocess.check_output([OBJDUMP, "-t", code[0]], cwd=tmp_path, text=True)
    names = sorted({m.group(1) for m in re.finditer(r"(\S+)\.kd$", out, re.M)})
    text = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True, check=True).stdout
    assert names

    def short(n):
        n = n.replace("(anonymous namespace)::", "").replace("incvit::", "").replace("void ", "").split("(")[0]
        return re.sub(r"\s+", "", n).replace("unsignedshort", "bf16")

    return {short(n) for n in text.splitlines()}


def sweep():
    """Calls over the documented ranges."""
    rows = [1, 8, 20, 40, 130, 200, 500, 700, 1000, 1024, 2048, 2050, 4300]
    for dtype in ("bf16", "f32"):
        for residual in (False, True):
            for m in rows:
                for K in (70, 1152, 2200, 6200):
                    for N in (65, 64, 808, 1144, 1145, 2001, 2040, 4088, 4304, 4305):
                        yield linear(dtype, m, K, N, residual)
            yield linear(dtype, 4090, 70, 4088, residual)
        for d in range(2, 258, 2):
            for rot in sorted({0, 2, d // 2 // 2 * 2, d}):
                for m in (1, 70000):
                    yield "qk", dict(dtype=dt(dtype), rows=m, hq=4, hk=2, d=d, rot=rot)
        yield "qk", dict(dtype=dt(dtype), rows=5, hq=4, hk=2, d=64, rot=64, off=2 if dtype == "bf16" else 4)
        for K in (64, 65, 1025, 1152, 2049, 2056, 6200, 6201):
            yield "quantize", dict(dtype=dt(dtype), rows=30, K=K)
        for K in (64, 65, 2056, 6200, 3001):
            for N in (64, 65):
                yield linear(dtype, 3, K, N)
                yield linear(dtype, 3, K, N, True)
        for B, dim, heads, mlp in [(b, *s) for b in (1, 2, 3, 4, 8, 10, 17, 32, 33)
                                   for s in ((96, 3, 100), (320, 10, 4096), (1024, 16, 300), (1024, 8, 4096), (1152, 16, 450), (2048, 16, 100))]:
            yield full(large.shape(dim, heads, mlp, dtype=dtype), B)
        for dim, heads in ((128, 8), (192, 8), (192, 4), (448, 8), (384, 4), (256, 2), (576, 8), (128, 1), (64, 8)):
            for B in (1, 33):
                yield full(large.shape(dim, heads, 100, dtype=dtype), B)
        for side, B in ((12, 1), (24, 1), (48, 1), (54, 2), (60, 3), (96, 1), (96, 2)):
            for mlp in (64, 600, 2200, 4304):
                yield full(large.shape(1152, 16, mlp, side=side, dtype=dtype), B)
                yield full(large.shape(2048, 16, mlp, side=side, dtype=dtype), B)


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump not installed")
def test_every_kernel_of_the_operators_is_launched_by_some_call(tmp_path):
    calls = list(sweep())
    reached = {e[0] for entries in launches(calls, tmp_path) for e in entries}
    built = compiled(tmp_path, "k_qk.hip") | compiled(tmp_path, "k_qlinear.hip")
    built = {b for b in built if not b.startswith(("q_scale", "q_pack"))}  # weights: one instance for each type
    assert sorted(built - reached) == []

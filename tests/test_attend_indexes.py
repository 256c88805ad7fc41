"""Index arithmetic that the attention kernels share, on the CPU: the functions are compiled for the host and looked at over all
sizes that calls may have."""
import os
import subprocess

import pytest

from paper_2607_12287_amd import build as hip_build

pytestmark = pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")


def run_on_host(tmp_path, header, body):
    """Compiles `body` as main behind `header` with host code only, and runs it; it prints what it finds wrong."""
    src, exe = tmp_path / "host.hip", str(tmp_path / "host")
    src.write_text('#include "%s"\n#include <cstdio>\n#include <random>\nusing namespace incvit;\nint main() {\n%s\n}\n' % (header, body))
    subprocess.check_call([hip_build.HIPCC, *hip_build.COMMON, "-O1", "--offload-host-only", str(src), "-o", exe])
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout == "", res.stdout[:2000] + res.stderr[-2000:]


def test_looking_for_infinities_stays_in_the_row(tmp_path):
    """A lane reads 4 dims from 16 k + 4 g on, of keys whose row has d of them, and what it reads for others lies in the row too."""
    run_on_host(tmp_path, "attend_plain.hpp", """
  for (int d = 8; d <= 256; d += 8)
    for (int k = 0; k < kv_dims(d) / 16; ++k)
      for (int g = 0; g < 4; ++g)
        for (int i = 0; i < 4; ++i) {
          const int at = special_dim(k, g, i, d);
          if (at < 0 || at >= d || (16 * k + 4 * g < d && at != 16 * k + 4 * g + i)) printf("d %d k %d g %d i %d: %d\\n", d, k, g, i, at);
        }""")

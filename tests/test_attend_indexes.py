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


def test_even_shares_are_no_more_than_the_launch_has(tmp_path):
    """As many as `even` and one for each sequence, also for the longest sequences (2^30 keys, 2^25 tiles)."""
    run_on_host(tmp_path, "attend.hpp", """
  std::mt19937 r(5);
  for (int trial = 0; trial < 200000; ++trial) {
    const int n = 1 + r() % kEvenTiles, even = 1 + r() % 1536, most = r() % 26;
    int nt[kEvenTiles];
    long total = 0;
    for (int i = 0; i < n; ++i) {
      nt[i] = trial % 7 == 0 ? 1 << most : (int)(r() % (1u << (r() % (most + 1)))) + (r() % 2);
      total += nt[i] < kEvenMost ? nt[i] : kEvenMost;
    }
    if (total != (int)total) printf("total %ld\\n", total);
    const int chunk = even_chunk((int)total, 16, even);
    long shares = 0;
    for (int i = 0; i < n; ++i) {
      const int c = even_count(nt[i], chunk);
      shares += c;
      if (c < 1 || c > kMostShares || (c < kMostShares && nt[i] <= kEvenMost && (long)c * chunk < nt[i])) printf("%d tiles: %d of %d\\n", nt[i], c, chunk);
    }
    if (shares > even + n) printf("%d sequences, %d: %ld\\n", n, even, shares);
  }""")

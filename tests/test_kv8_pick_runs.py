"""Which blocks of keys the waves of a search look up (host code of cg_kv8.h): all of them, and none
behind the last, whose place would be read from behind the page table."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

SRC = r"""
#include <cstdio>
#include <vector>
#include "cg_kv8.h"
int main() {
  int bad = 0, cases = 0;
  for (int waves : {4, 16})
    for (int n = 1; n <= 64 * 2100; n += n < 5000 ? 1 : 61) {
      const int blocks = (n + 63) / 64;
      std::vector<int> times(blocks, 0);
      int behind = 0;
      for (int w = 0; w < waves; ++w) {
        const PickRun r = pick_run(n, waves, w);
        for (int j = r.first; j < r.first + r.mine; ++j) {
          if (j >= 0 && j < blocks) ++times[j]; else ++behind;
        }
        for (int lane = 0; lane < 64; ++lane) {
          const int b = pick_block(r, lane);
          if (b >= blocks || b < -1) ++behind;
        }
      }
      for (int t : times) behind += t != 1;
      if (behind) { if (!bad) printf("waves %d, %d keys\n", waves, n); ++bad; }
      ++cases;
    }
  printf("%d cases, %d bad\n", cases, bad);
  return bad != 0 || cases < 5000;
}
"""


@pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which(HIPCC)), reason="no hipcc")
def test_no_wave_looks_behind_the_last_block(tmp_path):
    src = tmp_path / "runs.hip"
    src.write_text(SRC)
    exe = tmp_path / "runs"
    subprocess.run([HIPCC, "--offload-host-only", "-std=c++17", "-O1", "-w", "-I",
                    os.path.join(ROOT, "paper_2310_07240_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-2000:]

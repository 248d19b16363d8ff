"""The order of workgroups in attention over packed prompts (csrc/packed_order.h): every tile and
head has one workgroup, and a workgroup without one leaves.  Built with g++ from the header alone and run on the CPU."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_14586_amd", "csrc")

DRIVER = r'''
#include <cstdio>
#include <vector>
#include "packed_order.h"
int main() {
  long calls = 0;
  for (int H = 1; H <= 600; ++H)
    for (int total = 0; total * H <= 1300; ++total) {
      const int all = total * H;
      // as many as there are, a prompt more, and far more: the launch counts tiles that there may be
      for (int launched : {all, all + H, 2 * all + 3 * H, all + 1000}) {
        std::vector<int> taken(all);
        for (int wg = 0; wg < launched; ++wg) {
          const int r = vla::packed_rank(wg, total, H, [&](int n) { return n / H; });
          if (r >= all || (r < 0 && wg < all)) { std::printf("H %d total %d wg %d of %d: rank %d\n", H, total, wg, launched, r); return 1; }
          if (r >= 0 && taken[r]++) { std::printf("H %d total %d wg %d of %d: rank %d again\n", H, total, wg, launched, r); return 1; }
        }
        for (int r = 0; r < all; ++r)
          if (!taken[r]) { std::printf("H %d total %d of %d: rank %d left out\n", H, total, launched, r); return 1; }
        ++calls;
      }
    }
  std::printf("ok %ld\n", calls);
  return 0;
}
'''


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_tile_has_one_workgroup(tmp_path):
    src = tmp_path / "order_driver.cpp"
    src.write_text(DRIVER)
    exe = tmp_path / "order_driver"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout + r.stderr

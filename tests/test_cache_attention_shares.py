"""Where the combine of the cache attention reads, on the CPU: whatever stands in the workspace in
the place of a sequence's first and last CTA (a launch whose waits ran out leaves it unwritten), the
rows read lie within the workspace; and what the CTAs write is what is read."""
import os
import shutil
import subprocess

import pytest

SOURCE = r"""
#include "cache_attention.cuh"
#include <stdio.h>
using namespace ssd;
int main() {
  long checked = 0, none = 0;
  for (int B : {1, 7})
    for (int per_head : {B, B + 1, 19, 228})
      for (int group_rows : {8, 16})
        for (int row_groups : {1, 3})
          for (int Hkv : {1, 4}) {
            CacheAttnLaunch L{};
            L.per_head = per_head;
            L.row_groups = row_groups;
            L.group_rows = group_rows;
            const int64_t slots = per_head + B, room = (int64_t)Hkv * row_groups * slots * group_rows;
            const int odd[] = {-2147483647 - 1, -1, 0, 1, per_head / 2, per_head - 1, per_head,
                               2139062143, 2147483647};
            for (int b = 0; b < B; ++b)
              for (int x : odd)
                for (int y : odd)
                  for (int g = 0; g < Hkv; ++g)
                    for (int row = 0; row < row_groups * group_rows; ++row) {
                      const CacheShares s = cache_shares(L, B, b, make_int2(x, y), g, row);
                      const bool range = 0 <= x && x <= y && y < per_head;
                      if (s.parts != (range ? y - x + 1 : 0)) return printf("parts\n"), 1;
                      if (!range) {
                        ++none;
                        continue;
                      }
                      for (int i = 0; i < s.parts; ++i) {
                        const int64_t at = s.at + (int64_t)i * group_rows;
                        if (at < 0 || at >= room) return printf("outside\n"), 1;
                        // CTA (x + i, g, z) writes its row r of sequence b at this place
                        const int z = row / group_rows, r = row % group_rows;
                        if (at != (((int64_t)g * row_groups + z) * slots + x + i + b) * group_rows + r)
                          return printf("place\n"), 1;
                      }
                      ++checked;
                    }
          }
  printf("ok %ld %ld\n", checked, none);
  return checked > 0 && none > 0 ? 0 : 1;
}
"""


def test_shares_lie_within_the_workspace(tmp_path):
    from paper_2606_20543_gb300 import build
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    src, exe = tmp_path / "shares.cu", tmp_path / "shares"
    src.write_text(SOURCE)
    subprocess.run([build.nvcc()] + build.ARCH + ["-std=c++17", "-I" + build.CSRC,
                    "-I" + os.path.join(build.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout

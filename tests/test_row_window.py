"""The position table of the four-wave attention on the host: over parts of one to several windows, every step's
look-up lies inside the table, and every tile of the part is looked up once the window holds it."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "row_window.h"
using namespace infllm;
int main() {
  long looked = 0, moved = 0;
  for (int window : {16, 128})
    for (int t_begin : {0, 1, 57})
      for (int n = 1; n <= 3 * window + 9; ++n) {
        const int t_end = t_begin + n;
        int w0 = t_begin;
        auto look = [&](int tile) {  // as the kernel does: tile's entries, from the window's first
          const int at = offsets_tile(tile, t_end);
          ++looked;
          if (at >= w0 && at < w0 + window && (at == tile || tile >= t_end)) return true;
          std::printf("window %d part [%d, %d): tile %d in [%d, %d)\n", window, t_begin, t_end, at, w0, w0 + window);
          return false;
        };
        for (int t = t_begin; t < t_begin + kRowsAhead; ++t)  // the prologue
          if (!look(t)) return 1;
        for (int t = t_begin; t < t_end; ++t) {
          if (window_moves(t, t_end, w0, window)) {
            w0 = t + kRowsAhead;
            ++moved;
          }
          if (!look(t + kRowsAhead)) return 1;
        }
      }
  std::printf("%ld %ld\n", looked, moved);
  return looked > 10000 && moved > 300 ? 0 : 2;
}
"""


def test_row_window(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    (tmp_path / "window.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "window")
    subprocess.run([cxx, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I",
                    os.path.join(ROOT, "paper_2402_04617_amd", "csrc"), str(tmp_path / "window.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout

"""No GPU: up to which tables flashmask_decode keeps sequences whole (fm_cache_index.h), compiled for the host: on the side that was faster at
points where both were timed on an MI355X, for both head dimensions, 16- and 8-bit caches, heads stored side by side, and 1 to 1024 query rows to a head."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_01359_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "fm_cache_index.h"

// groups of 16 keys of a team's step, workgroups of a whole call, groups of a chunk at least, keys of a row of the table, us whole, us split
struct Timed {
  int round, workgroups, least, keys;
  double whole, split;
};
const Timed timed[] = {
    {8, 8, 8, 384, 8.7, 9.9}, {8, 8, 8, 640, 10.8, 9.9}, {8, 8, 8, 1024, 14.7, 9.9}, {8, 32, 8, 384, 8.9, 10.3},
    {8, 32, 8, 768, 11.8, 10.3}, {8, 128, 8, 320, 8.8, 11.7}, {8, 128, 8, 640, 12.8, 16.4}, {8, 128, 8, 768, 14.1, 17.6},
    {8, 512, 8, 1024, 44.8, 47.4}, {8, 512, 8, 768, 24.5, 27.6}, {16, 8, 8, 384, 8.6, 10.5}, {16, 8, 8, 512, 8.6, 10.9},
    {16, 8, 8, 768, 10.0, 10.9}, {16, 32, 8, 512, 9.4, 11.3}, {16, 32, 8, 768, 9.8, 11.4}, {16, 128, 8, 512, 8.8, 11.4},
    {16, 128, 8, 1024, 12.5, 14.9}, {16, 8, 8, 448, 9.4, 11.2}, {16, 8, 8, 512, 9.4, 11.3}, {16, 8, 8, 1024, 12.7, 11.4},
    {16, 128, 8, 512, 9.7, 11.7}, {16, 128, 8, 1024, 14.1, 15.3}, {32, 32, 8, 512, 9.0, 11.2}, {32, 32, 8, 768, 11.8, 12.6},
    {32, 512, 8, 1024, 20.8, 22.5}, {8, 4, 8, 384, 9.7, 10.6}, {8, 4, 8, 512, 11.1, 10.7}, {8, 4, 8, 640, 12.3, 10.7},
    {8, 256, 8, 1024, 21.0, 28.0}, {4, 8, 32, 384, 16.5, 18.9}, {4, 8, 32, 512, 18.8, 21.2}, {4, 8, 32, 768, 23.5, 20.8},
    {4, 512, 32, 1024, 47.9, 66.8}, {4, 256, 128, 512, 20.4, 25.7}, {4, 256, 128, 1024, 31.1, 37.3},
    {8, 256, 128, 1024, 25.7, 31.3}, {16, 8, 16, 384, 12.5, 14.0}, {16, 8, 16, 1024, 16.5, 14.1},
};

int main() {
  int wrong = 0;
  for (const Timed& t : timed) {
    const bool whole = t.keys <= fm_whole_keys(t.round, t.workgroups, t.least, 256);
    if (whole != (t.whole < t.split)) std::printf("%d %d %d %d\n", t.round, t.workgroups, t.least, t.keys), ++wrong;
  }
  // never a split of what cannot be split, nor beyond 32 bits
  for (int round : {4, 8, 16, 32})
    for (int least : {8, 128, 4096})
      for (long long workgroups : {1ll, 1000ll, 1ll << 30})
        for (int cus : {0, 1, 256}) {
          const long long line = fm_whole_keys(round, workgroups, least, cus);
          if (line < 16ll * least || line > 65536) ++wrong;
        }
  if (!wrong) std::printf("ok\n");
}
"""


def test_the_line_lies_where_measurements_meet(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("g++ not available")
    source, out = tmp_path / "check.cpp", str(tmp_path / "check")
    source.write_text(PROGRAM)
    subprocess.run([compiler, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(source), "-o", out],
                   check=True, timeout=120)
    done = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout + done.stderr

"""No GPU: how many rows the bounds of a key leave (fm_cache_index.h), compiled for the host, against a loop over the rows: for every two intervals with
ends in and around the rows and at the ends of 32 bits, without an overflow on the way."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_01359_amd", "csrc")

PROGRAM = r"""
#include <climits>
#include <cstdio>
#include <vector>
#include "fm_cache_index.h"

int main() {
  for (int lo : {-256, -3, 0, 1, 7, 199, (1 << 30) - 2, INT_MAX - 5})
    for (int rows : {-1, 0, 1, 2, 5}) {
      const int hi = lo + rows;
      std::vector<int> ends = {INT_MIN, INT_MIN + 1, INT_MIN / 2, -1, 0, 1, 200, 1 << 30, INT_MAX - 1, INT_MAX};
      for (long long i = lo - 2ll; i <= hi + 2ll; ++i)
        if (i <= INT_MAX) ends.push_back((int)i);
      for (int lts : ends)
        for (int lte : ends)
          for (int uts : ends)
            for (int ute : ends) {
              int want = 0;
              for (int i = lo; i < hi; ++i) want += !((lts <= i && i < lte) || (uts <= i && i < ute));
              const int got = fm_rows_left(lo, hi, lts, lte, uts, ute);
              if (got != want) {
                std::printf("rows [%d, %d), bounds %d %d %d %d: %d for %d\n", lo, hi, lts, lte, uts, ute, got, want);
                return 1;
              }
            }
    }
  std::printf("ok\n");
}
"""


def test_rows_left_against_a_loop(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("g++ not available")
    source, out = tmp_path / "check.cpp", str(tmp_path / "check")
    source.write_text(PROGRAM)
    subprocess.run([compiler, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(source), "-o", out],
                   check=True, timeout=120)
    done = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout + done.stderr

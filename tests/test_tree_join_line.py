"""No GPU: which of its two joins a call on trees of many rows takes (fm_cache_index.h), compiled for the host: the one that was faster, or within a tenth of it, at
points where both were timed on an MI355X: both head dimensions, 1 to 64 sequences, 128 to 8064 rows, 8 to 256 chunks."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_01359_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include "fm_cache_index.h"

// rows of all heads, sequences, chunks, keys of a row of the table, us by a workgroup to a row, us by a few lanes to a row
struct Timed {
  int rows, sequences, chunks, keys;
  double workgroups, lanes;
};
const Timed timed[] = {
    {2016, 16, 32, 8192, 16.2, 6.2}, {1024, 16, 64, 8192, 13.6, 7.1}, {512, 16, 64, 8192, 7.9, 5.0}, {504, 16, 128, 8192, 9.6, 7.5}, {128, 16, 256, 8192, 5.1, 11.0},
    {8064, 16, 16, 8192, 48.6, 11.9}, {2048, 16, 16, 8192, 14.9, 5.5}, {2016, 1, 32, 8192, 7.8, 9.4}, {1024, 1, 64, 8192, 8.3, 15.1}, {512, 1, 64, 8192, 4.9, 15.6},
    {504, 1, 128, 8192, 4.7, 14.7}, {128, 1, 256, 8192, 3.8, 14.0}, {8064, 1, 8, 8192, 10.0, 7.3}, {2048, 1, 16, 8192, 5.7, 6.0}, {2016, 4, 32, 2048, 10.2, 6.8},
    {1024, 4, 64, 2048, 8.2, 7.5}, {512, 4, 64, 2048, 4.9, 5.6}, {504, 4, 128, 2048, 4.6, 5.4}, {128, 4, 256, 2048, 3.9, 5.2}, {8064, 4, 8, 2048, 24.0, 8.5},
    {2048, 4, 16, 2048, 9.3, 4.7}, {2016, 1, 32, 100032, 7.9, 11.4}, {1024, 1, 64, 100032, 9.3, 16.6}, {512, 1, 64, 100032, 5.6, 16.0}, {504, 1, 128, 100032, 7.5, 26.5},
    {128, 1, 256, 100032, 6.9, 47.0}, {8064, 1, 8, 100032, 11.3, 8.3}, {2048, 1, 16, 100032, 6.1, 7.3}, {2016, 64, 64, 1536, 44.2, 10.2}, {1024, 64, 64, 1536, 28.2, 8.0},
    {512, 64, 64, 1536, 15.5, 5.1}, {504, 64, 128, 1536, 17.6, 5.7}, {128, 64, 256, 1536, 7.2, 4.6}, {2048, 64, 32, 1536, 37.9, 8.3}, {2016, 40, 64, 3008, 27.4, 7.2},
    {1024, 40, 64, 3008, 18.4, 5.7}, {512, 40, 64, 3008, 10.5, 4.4}, {504, 40, 128, 3008, 15.0, 7.2}, {128, 40, 256, 3008, 6.2, 6.0}, {2048, 40, 32, 3008, 30.1, 7.8},
    {2016, 16, 32, 8192, 21.3, 5.0}, {1024, 16, 64, 8192, 16.4, 5.0}, {512, 16, 64, 8192, 9.3, 4.5}, {504, 16, 128, 8192, 10.7, 6.6}, {128, 16, 256, 8192, 4.8, 11.0},
    {8064, 16, 16, 8192, 62.1, 7.8}, {2048, 16, 16, 8192, 17.7, 4.2}, {2016, 1, 32, 8192, 5.9, 8.5}, {1024, 1, 64, 8192, 5.1, 14.6}, {512, 1, 64, 8192, 4.0, 14.8},
    {504, 1, 128, 8192, 4.0, 14.3}, {128, 1, 256, 8192, 2.6, 14.3}, {8064, 1, 8, 8192, 11.6, 5.0}, {2048, 1, 16, 8192, 5.2, 5.4}, {2016, 4, 32, 2048, 11.4, 4.8},
    {1024, 4, 64, 2048, 7.1, 5.6}, {512, 4, 64, 2048, 4.4, 5.1}, {504, 4, 128, 2048, 4.6, 5.3}, {128, 4, 256, 2048, 2.7, 5.2}, {8064, 4, 8, 2048, 36.3, 5.2},
    {2048, 4, 16, 2048, 10.6, 4.0}, {2016, 1, 32, 100032, 6.3, 8.8}, {1024, 1, 64, 100032, 6.0, 15.0}, {512, 1, 64, 100032, 4.7, 15.5}, {504, 1, 128, 100032, 5.4, 26.4},
    {128, 1, 256, 100032, 4.7, 46.0}, {8064, 1, 8, 100032, 11.7, 5.7}, {2048, 1, 16, 100032, 5.6, 5.8}, {2016, 64, 64, 1536, 67.9, 7.8}, {1024, 64, 64, 1536, 35.8, 5.0},
    {512, 64, 64, 1536, 19.8, 4.4}, {504, 64, 128, 1536, 23.1, 4.3}, {128, 64, 256, 1536, 9.1, 4.0}, {2048, 64, 32, 1536, 42.5, 5.1}, {2016, 40, 64, 3008, 45.1, 5.7},
    {1024, 40, 64, 3008, 24.3, 4.4}, {512, 40, 64, 3008, 13.6, 4.2}, {504, 40, 128, 3008, 19.8, 4.9}, {128, 40, 256, 3008, 7.4, 5.5}, {2048, 40, 32, 3008, 34.2, 5.0},
};

int main() {
  int wrong = 0;
  for (const Timed& t : timed) {
    const bool lanes = fm_tree_joins_by_lanes(t.rows, t.sequences, t.chunks, 8, t.keys);
    const double taken = lanes ? t.lanes : t.workgroups, other = lanes ? t.workgroups : t.lanes;
    if (taken > 1.1 * other) std::printf("%d %d %d %d: %.1f us, the other %.1f\n", t.rows, t.sequences, t.chunks, t.keys, taken, other), ++wrong;
  }
  // the largest calls
  if (!fm_tree_joins_by_lanes(1 << 24, 64, 1, 8, 1 << 30)) ++wrong;
  if (fm_tree_joins_by_lanes(64, 1, 256, 8, 1 << 30)) ++wrong;
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

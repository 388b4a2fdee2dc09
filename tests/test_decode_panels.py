"""No GPU: how flashmask_decode goes through a chunk's keys (fm_cache_index.h), compiled for the host: every key lies in exactly one panel,
and every panel begins where a group of 16 keys does, up to the longest row that a table may have."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_01359_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "fm_cache_index.h"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  const int most = 1 << 30;   // keys of a row of the table
  for (int keys : {0, 2048})
    for (int begin : {0, 16, 2032, most - 4096, most - 2048, most - 16, most})
      for (int end : {0, 1, 16, 2047, 2048, 2049, 100000, most / 2 - 1, most / 2, most - 2049, most - 1, most}) {
        int upto = begin, panels = 0;   // where the panels before have ended
        for (int panel = begin; panel < end; panel = fm_next_panel(panel, end, keys)) {
          CHECK(panel == upto && panel % FM_KEY_GROUP == 0);
          upto = keys > 0 && end - panel > keys ? panel + keys : end;   // what the kernel takes of it
          ++panels;
        }
        CHECK(upto == (begin < end ? end : begin));
        CHECK(keys > 0 || panels == (begin < end ? 1 : 0));
      }
  std::printf("ok\n");
}
"""


def test_panels_cover_every_key_once(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("g++ not available")
    source, out = tmp_path / "check.cpp", str(tmp_path / "check")
    source.write_text(PROGRAM)
    subprocess.run([compiler, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(source), "-o", out],
                   check=True, timeout=120)
    done = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout + done.stderr

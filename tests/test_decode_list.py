"""No GPU: the list of a call's chunks (fm_cache_index.h), compiled for the host: units, partial results and split sequences stay within the
arrays that the scratch has for them, and the chunks of a sequence cover its keys once, up to 65535 sequences."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_01359_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <vector>
#include "fm_cache_index.h"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  std::srand(7);
  for (int trial = 0; trial < 1500; ++trial) {
    const int B = trial < 20 ? 65535 - trial : 1 + std::rand() % (trial % 2 ? 3000 : 300);
    const int chunks = 1 + std::rand() % 256, step = 2 << std::rand() % 3, round = step * (1 + std::rand() % 4), least = 8 << std::rand() % 8;
    const int kind = std::rand() % 4;   // all short, one long, some long, all alike
    const int longest = 1 + std::rand() % 4000;
    std::vector<int> groups(B);
    unsigned total = 0;
    for (int b = 0; b < B; ++b) {
      groups[b] = kind == 3 ? longest : (kind == 1 ? b == B / 2 : kind == 2 && std::rand() % 8 == 0) ? std::rand() % (kind == 1 ? 1 << 22 : longest) : std::rand() % 4;
      total += groups[b];
    }
    const int size = fm_chunk_groups(total, fm_divisor(chunks), least, round);
    long long units = 0, slots = 0, splits = 0;
    for (int g : groups) {
      const int n = fm_chunks_of(g, size);
      CHECK(n < 1 << 15);   // chunk and chunks share a word
      units += n;
      if (n > 1) {
        slots += n;
        ++splits;
        const int even = fm_even_chunk(g, n, step);
        long long upto = 0;
        for (int c = 0; c < n; ++c) {
          const long long from = (long long)c * even, to = from + even < g ? from + even : g;
          if (from < g) { CHECK(from == upto); upto = to; }
        }
        CHECK(upto == g);
      }
    }
    CHECK(units <= fm_most_units(chunks, B) && units <= fm_listed_units(chunks, B) && fm_listed_units(chunks, B) % 8 == 0);
    CHECK(slots <= fm_most_slots(chunks, B));
    CHECK(splits <= fm_most_splits(chunks, B));
  }
  std::printf("ok\n");
}
"""


def test_the_list_stays_within_its_arrays(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("g++ not available")
    source, out = tmp_path / "check.cpp", str(tmp_path / "check")
    source.write_text(PROGRAM)
    subprocess.run([compiler, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(source), "-o", out],
                   check=True, timeout=120)
    done = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout + done.stderr

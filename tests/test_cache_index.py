"""No GPU: the kernels' integer code for the paged cache (fm_cache_index.h), compiled for the host: no index value is followed out of
its range, every key that a row can see lies in exactly one chunk, chunks and partial results stay within what the launch
and its scratch have room for, and a fork's row is what the definition says."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_01359_amd", "csrc")

PROGRAM = r"""
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "fm_cache_index.h"

#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

int main() {
  for (int entry : {INT_MIN, -2, -1, 0, 1, 6, 7, 8, INT_MAX}) CHECK(fm_known_page(entry, 7) == (entry >= 0 && entry < 7 ? entry : -1));
  for (int page : {16, 32, 48, 64, 112, 256, 1 << 20})
    for (int columns : {1, 2, 17})
      for (int position : {INT_MIN, -1, 0, 1, page - 1, page, page + 1, page * columns - 1, page * columns, INT_MAX}) {
        const FmPlace p = fm_place(position, fm_divisor(page), columns);
        if (position < 0 || position / page >= columns) CHECK(p.column == -1);
        else CHECK(p.column == position / page && p.slot == position % page);
      }
  // what a row sees lies in the range, and the range in the table
  for (int len : {INT_MIN, -1, 0, 1, 2, 5, 15, 16, 17, 40, 63, 64, 65, 100, INT_MAX})
    for (int T : {1, 2, 5, 8, 70})
      for (int window : {0, 1, 2, 16, 17, 33, (1 << 30) - 1})
        for (int table_keys : {16, 48, 64, 112}) {
          const FmKeyRange r = fm_key_range(len, T, window, table_keys);
          CHECK(r.lo >= 0 && r.lo <= r.hi && r.hi <= table_keys && r.lo % FM_KEY_GROUP == 0 && r.len == (len > 0 ? len : 0));
          for (int t = 0; t < T; ++t)
            for (int j = 0; j < table_keys && j < r.len; ++j) {
              const long long i = (long long)r.len - T + t;
              if (j <= i && (window == 0 || j > i - window)) CHECK(j >= r.lo && j < r.hi);
            }
        }
  // chunks, as the kernel deals them
  std::srand(5);
  for (int trial = 0; trial < 20000; ++trial) {
    const int B = 1 + std::rand() % 40, chunks = 1 + std::rand() % (trial % 3 ? 40 : 300), round = 8 << std::rand() % 4;
    const long long most = 1ll << std::rand() % 24;
    std::vector<int> groups(B);
    unsigned total = 0;
    for (int& g : groups) total += g = std::rand() % 5 ? (int)(((long long)std::rand() << 10 ^ std::rand()) % most) : 0;
    const int least = 8 << std::rand() % 4, size = fm_chunk_groups(total, fm_divisor(chunks), least, round);
    CHECK(size % round == 0 && size >= least);
    long long units = 0, slots = 0;
    for (int g : groups) {
      const int n = fm_chunks_of(g, size);
      CHECK(n >= 1 && (long long)n * size >= g && (n == 1 || (long long)(n - 1) * size < g));
      units += n;
      slots += n > 1 ? n : 0;
      for (int steps : {2, 4, 8})   // groups of a wave's step; a round is a multiple of it
        if (round % steps == 0 && n > 1) {
          const int even = fm_even_chunk(g, n, steps);
          CHECK(even % steps == 0 && even <= size && (long long)n * even >= g && (long long)(n - 1) * even * 16 <= INT_MAX);
        }
    }
    CHECK(units <= fm_most_units(chunks, B));
    CHECK(slots <= fm_most_slots(chunks, B));
  }
  CHECK(fm_chunk_groups(1u << 30, fm_divisor(1), 8, 64) >= 1 << 30);
  for (int page : {16, 48, 64})
    for (int len : {INT_MIN, -1, 0, 1, 15, 16, 17, 48, 95, 96, 128, INT_MAX}) {
      const FmFork f = fm_fork(len, fm_divisor(page));
      const int have = len > 0 ? len : 0;
      CHECK(f.last == have / page && f.partly == (have % page != 0));
      for (int c = 0; c < 9; ++c) {
        CHECK(fm_fork_entry(f, c, 40 + c, -1) == 40 + c);
        CHECK(fm_fork_entry(f, c, 40 + c, 7) == (c < have / page ? 40 + c : c == have / page && have % page ? 7 : -1));
      }
    }
  std::printf("ok\n");
}
"""


def test_index_arithmetic(tmp_path):
    compiler = shutil.which("g++")
    if not compiler:
        pytest.skip("g++ not available")
    source = tmp_path / "check.cpp"
    source.write_text(PROGRAM)
    out = str(tmp_path / "check")
    subprocess.run([compiler, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(source), "-o", out],
                   check=True, timeout=120)
    done = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout + done.stderr

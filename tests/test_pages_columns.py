"""Which entries the query tokens of attention of several tokens see, for lengths of any value: the functions that the kernel uses
(csrc/pages_columns.h), compiled for the CPU, against the same in 64 bits (no GPU needed)."""
from __future__ import annotations

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include "pages_columns.h"

int main() {
  const int32_t low = INT32_MIN, high = INT32_MAX;
  const int32_t lens[] = {low, low + 1, low + 31, low + 32, low + 63, low + (1 << 28) - 1, -(1 << 28), -65, -64, -1, 0, 1, 63, 64, 65, 100000, 0x7FFF0000, high};
  const int32_t bounds[] = {1, 7, 64, 131072, 0x7FFF0000};
  const int32_t tokens[] = {1, 2, 33, 64, 65, 4097, (1 << 28) - 1};
  long wrong = 0, outside = 0;
  for (int32_t max_len : bounds)
    for (int32_t len : lens)
      for (int32_t m : tokens)
        for (int32_t token : {0, m / 3, m / 2, m - 1}) {
          const int64_t n = std::min(std::max(int64_t(len), int64_t(0)), int64_t(max_len));
          const int64_t want = std::max(n - m + token, int64_t(-1));
          const int32_t got = d2o::last_seen(d2o::entries_of(len, max_len), m, token);
          wrong += got != want;
          outside += got < -1 || got >= max_len;  // (an entry behind the last one that the page table's row names)
        }
  long shares = 0;
  for (int32_t max_len : bounds)
    for (int32_t window : {1, 64, high})
      for (int32_t sink : {0, 4, high - 32, high - 31, high})
        for (int32_t columns : {0, 32}) {
          const __int128 all = (__int128(max_len) + 15) / 16, shown = (__int128(window) + sink + columns) / 16 + 3;
          shares += d2o::shown_tiles(max_len, window, sink, columns, 16) != (shown < all ? shown : all);
        }
  printf("%ld %ld %ld\n", wrong, outside, shares);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("columns")
    src = where / "columns.cpp"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2406_13035_amd", "csrc"), "-o", str(where / "columns"), str(src)],
                   check=True)
    return str(where / "columns")


def counts(program):
    return list(map(int, subprocess.run([program], check=True, capture_output=True, text=True).stdout.split()))


def test_lengths_of_any_value(program):
    wrong, outside, _ = counts(program)
    assert outside == 0 and wrong == 0


def test_first_tokens_up_to_the_largest_number(program):
    assert counts(program)[2] == 0

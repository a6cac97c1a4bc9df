"""The decode kernels' own arithmetic of key ranges and 4-bit value loads (csrc/key_ranges.hpp), compiled for the host: every
length and split count, and every load of every tile that a workgroup works on."""
import os
import subprocess

import pytest

from conftest import ROOT

PROGRAM = r"""
#include "key_ranges.hpp"
#include <cstdio>
#include <cstdlib>
#include <set>
using namespace potattn;

#define CHECK(x, ...) do { if (!(x)) { std::printf("%s: ", #x); std::printf(__VA_ARGS__); std::printf("\n"); std::exit(1); } } while (0)

// The tiles that a workgroup of `waves` waves loads from: each wave's first, and the next one ahead of its use (past the
// range: the last again), as the kernel's loops do. A workgroup without tiles loads nothing.
static void tiles_loaded(const KeyRange& r, int waves, std::set<int>& got) {
  got.clear();
  for (int w = 0; w < waves; ++w)
    for (int j = w; j < r.tiles; j += waves) {
      got.insert(j);
      got.insert(j + waves < r.tiles - 1 ? j + waves : r.tiles - 1);
    }
}

static long tiles_checked = 0;
static void check_loads(int t_all, const KeyRange& r) {
  const int t_cap = (t_all + 7) / 8 * 8;  // the tightest cache
  std::set<int> tiles;
  for (int waves : {4, 12, 16}) {
    tiles_loaded(r, waves, tiles);
    CHECK((r.tiles <= 0) == tiles.empty(), "t_all %d", t_all);
    if (tiles.empty()) continue;
    const int last = groups_end(r);
    CHECK(last <= t_cap && last % 8 == 0 && last >= r.end, "t_all %d end %d", t_all, r.end);
    for (int j : tiles) {
      const int t0 = r.begin + kWTile * j;
      CHECK(j >= 0 && t0 >= r.begin && t0 < r.end, "t_all %d tile %d", t_all, j);
      const long window = (long)(last - t0) * (kI4GroupBytes / 8);  // bytes from the tile's first group
      CHECK(t0 % 8 == 0 && window > 0, "t0 %d", t0);
      ++tiles_checked;
      for (int lane = 0; lane < 64; ++lane) {
        const int at[4] = {value_offset_i4(lane, 0), value_offset_i4(lane, 1), step_offset_i4(lane),
                           step_offset_i4(lane) + kI4Minima - kI4Steps};
        for (int a : at) CHECK(a >= 0 && a % 16 == 0 && (a + 16 <= window || a >= window), "t0 %d lane %d", t0, lane);
      }
    }
  }
}

int main() {
  // what a lane's loads hold: its 8 tokens of K-block kb, and the 8 keys whose weights it forms
  for (int lane = 0; lane < 64; ++lane) {
    for (int kb = 0; kb < 2; ++kb)
      CHECK(value_offset_i4(lane, kb) == ((32 * kb + 8 * (lane / 16)) / 8) * kI4GroupBytes + 16 * (lane % 16), "lane %d", lane);
    const int first = 32 * (lane / 8 % 2) + 8 * (lane / 16);
    CHECK(step_offset_i4(lane) == first / 8 * kI4GroupBytes + 256, "lane %d", lane);
  }
  static_assert(kI4Minima == kI4Steps + 16 && kI4GroupBytes == 288, "record");
  // a length per sequence: the ranges are the sequence in order, and one of them takes the appended token in
  for (int n_splits = 1; n_splits <= 72; ++n_splits)
    for (int t_all = 0; t_all <= 6000; t_all += t_all < 1300 ? 1 : 61) {
      const int len = own_split_len(t_all, n_splits);
      CHECK(len % kWTile == 0 && (long)len * n_splits >= t_all, "t_all %d n %d", t_all, n_splits);
      int next = 0, holders = 0;
      for (int s = 0; s < n_splits; ++s) {
        const KeyRange r = split_range(t_all, s, len);
        if (r.tiles > 0) {
          CHECK(r.begin == next && r.end > r.begin && r.begin % kWTile == 0, "t_all %d split %d", t_all, s);
          CHECK(r.tiles == (r.end - r.begin + 63) / 64, "t_all %d split %d", t_all, s);
          next = r.end;
        } else {
          CHECK(r.begin >= t_all, "t_all %d split %d", t_all, s);
        }
        if (holds_last(r, t_all)) {
          ++holders;
          CHECK(r.tiles > 0 && t_all - 1 >= r.begin && t_all - 1 < r.end, "t_all %d split %d", t_all, s);
        }
        if (t_all < 1300 || t_all % 7 == 0) check_loads(t_all, r);
      }
      CHECK(next == t_all && holders == (t_all > 0), "t_all %d n %d", t_all, n_splits);
    }
  // the longest sequences: no sum passes an int
  const int most = (1 << 24) - 8;
  for (int n_splits : {1, 3, 256, 2048}) {
    const int len = own_split_len(most, n_splits);
    const KeyRange r = split_range(most, n_splits - 1, len);
    CHECK(r.end <= most && (long)len * n_splits < (1L << 31), "n %d", n_splits);
    CHECK((long)most * (kI4GroupBytes / 8) < (1L << 31), "n %d", n_splits);
  }
  std::printf("%ld tiles\n", tiles_checked);
}
"""


def _run(tmp_path, program):
    source, binary = tmp_path / "ranges.cpp", tmp_path / "ranges"
    source.write_text(program)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I",
                    os.path.join(ROOT, "paper_2609_09208_amd", "csrc"), "-o", str(binary), str(source)], check=True)
    return subprocess.run([str(binary)], capture_output=True, text=True, timeout=300)


def test_ranges_and_loads(tmp_path):
    res = _run(tmp_path, PROGRAM)
    assert res.returncode == 0, res.stdout + res.stderr
    assert int(res.stdout.split()[0]) > 1000


@pytest.mark.parametrize("planted", [
    ("groups_end(r)", "(groups_end(r) + 8)"),                                # a window one group too long
    ("own_split_len(t_all, n_splits)", "(t_all + n_splits - 1) / n_splits"),  # ranges that are not whole tiles
    ("holds_last(r, t_all)", "(s == n_splits - 1)"),                         # the last split, empty or not
    ("value_offset_i4(lane, 1)", "(value_offset_i4(lane, 1) + 8)"),
])
def test_a_wrong_range_is_found(tmp_path, planted):
    assert planted[0] in PROGRAM
    res = _run(tmp_path, PROGRAM.replace(*planted))
    assert res.returncode == 1, res.stdout

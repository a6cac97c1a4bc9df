"""Tiles of tokens whose places lie past the keys that a call looks at (csrc/page_ranges.hpp), compiled for the host: a sequence may
be longer than max_len, and keys past max_len are not seen. Key by key, over places on both sides of the end."""
import os
import subprocess

from conftest import ROOT

PROGRAM = r"""
#include "page_ranges.hpp"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace potattn;
#define CHECK(x, ...) do { if (!(x)) { std::printf("%s: ", #x); std::printf(__VA_ARGS__); std::printf("\n"); std::exit(1); } } while (0)

// tokens p_first .. p_last, keys 0 .. len - 1
static void check(int p_first, int p_last, int len, int window, int n_sink) {
  const SeenTiles s = seen_tiles(p_first, p_last, len, window, n_sink);
  CHECK(s.sink_tiles >= 0 && s.tiles >= s.sink_tiles, "%d..%d of %d, window %d sinks %d: %d of %d tiles", p_first, p_last, len, window,
        n_sink, s.sink_tiles, s.tiles);
  std::vector<int> in(len + 64, 0);
  for (int j = 0; j < s.tiles; ++j) {
    const int t0 = tile_start(s, j);
    CHECK(t0 >= 0 && t0 % kWTile == 0 && t0 < s.end && s.end <= len, "%d..%d of %d, window %d sinks %d: tile %d at %d, end %d", p_first,
          p_last, len, window, n_sink, j, t0, s.end);
    bool all = true;
    for (int k = t0; k < t0 + kWTile; ++k) {
      ++in[k];
      for (int p = p_first; p <= p_last; ++p) all &= k < len && sees(p, k, window, n_sink);
    }
    const bool whole = whole_tile(s, p_first, p_last, t0, window, n_sink);
    CHECK(!whole || all, "%d..%d of %d, window %d sinks %d: tile at %d", p_first, p_last, len, window, n_sink, t0);
    // what is left to masks: the first and the last tiles of the runs
    if (window <= 0 && t0 + kWTile <= len && t0 + kWTile <= p_first) CHECK(whole, "%d..%d of %d: tile at %d", p_first, p_last, len, t0);
  }
  for (int k = 0; k < len; ++k) {
    bool seen = false;
    for (int p = p_first; p <= p_last; ++p) seen |= sees(p, k, window, n_sink);
    CHECK(in[k] <= 1 && (!seen || in[k] == 1), "%d..%d of %d, window %d sinks %d: key %d", p_first, p_last, len, window, n_sink, k);
  }
  for (int n : {1, 2, 7, 64}) {  // splits: every tile once
    int next = 0;
    for (int i = 0; i < n; ++i) {
      const TileRun r = split_tiles(s.tiles, i, n);
      CHECK(r.first == (next < s.tiles ? next : s.tiles) && r.end >= r.first && r.end <= s.tiles, "split %d of %d", i, n);
      next = r.end;
    }
    CHECK(next == s.tiles, "%d of %d", next, s.tiles);
  }
}

int main() {
  check(999, 999, 100, 50, 4);
  check(5199, 5199, 4096, 1000, 70);
  check(999, 999, 100, 0, 0);
  for (int len : {1, 7, 64, 65, 100, 128, 321, 700})
    for (int first : {-3, 0, 50, 63, 99, 100, 120, 127, 190, 400, 999, 5000})
      for (int n : {1, 2, 40, 200})
        for (int window : {0, 1, 50, 63, 64, 65, 200, 1000})
          for (int sinks : {0, 1, 4, 63, 64, 65, 70, 130, 1000}) check(first, first + n - 1, len, window, sinks);
  std::printf("ok\n");
}
"""


def test_no_key_past_the_end_is_seen(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "t")
    csrc = os.path.join(ROOT, "paper_2609_09208_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", csrc, "-o", exe, str(src)], check=True)
    got = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and got.stdout.strip() == "ok", got.stdout[-2000:]

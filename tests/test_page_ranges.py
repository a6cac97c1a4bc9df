"""The paged kernels' own arithmetic (csrc/page_ranges.hpp), compiled for the host: division by a page's groups, the tiles that
tokens see, and their split, against the definitions key by key."""
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

static void check_div(uint32_t d, uint32_t step) {
  const PageDiv v = page_div(d);
  for (uint32_t g = 0; g < (1u << 21); g += step) CHECK(page_of_group(g, v) == g / d, "%u / %u", g, d);
  for (uint32_t q = 1; q * (uint64_t)d < (1u << 21); ++q)  // both sides of every multiple
    CHECK(page_of_group(q * d, v) == q && page_of_group(q * d - 1, v) == q - 1, "%u %u", q, d);
  CHECK(page_of_group((1u << 21) - 1, v) == ((1u << 21) - 1) / d, "%u", d);
}

static void check_seen(int p_first, int p_last, int len, int window, int n_sink) {
  const SeenTiles s = seen_tiles(p_first, p_last, len, window, n_sink);
  std::vector<int> in(len + 200, 0);
  CHECK(s.tiles >= 0 && s.sink_tiles >= 0 && s.sink_tiles <= s.tiles, "%d", s.tiles);
  for (int j = 0; j < s.tiles; ++j) {
    const int t0 = tile_start(s, j);
    CHECK(t0 >= 0 && t0 % kWTile == 0 && t0 < s.end, "tile %d at %d, end %d", j, t0, s.end);
    bool all = true, none = true;
    for (int k = t0; k < t0 + kWTile; ++k) {
      ++in[k];
      for (int p = p_first; p <= p_last; ++p) (sees(p, k, window, n_sink) ? none : all) = false;
    }
    if (p_first >= 0) {
      CHECK(!all_seen(p_first, p_last, t0, window, n_sink) || all, "%d..%d t0 %d", p_first, p_last, t0);
      CHECK(!none_seen(p_first, p_last, t0, window, n_sink) || none, "%d..%d t0 %d", p_first, p_last, t0);
    }
  }
  for (int k = 0; k < len; ++k) {
    bool seen = false;
    for (int p = p_first; p <= p_last; ++p)
      seen |= k <= p && (window <= 0 || k > p - window || k < n_sink);
    CHECK(in[k] <= 1, "key %d in %d tiles", k, in[k]);
    CHECK(!seen || (in[k] == 1 && k < s.end), "key %d of %d, tokens %d..%d window %d sinks %d", k, len, p_first, p_last, window, n_sink);
  }
  CHECK(s.end <= len || len <= 0, "end %d", s.end);
  // splits: every tile once
  for (int n : {1, 2, 3, 7, 32, 64}) {
    int next = 0;
    for (int i = 0; i < n; ++i) {
      const TileRun r = split_tiles(s.tiles, i, n);
      CHECK(r.first <= r.end && r.first == (next < s.tiles ? next : s.tiles) && r.end <= s.tiles, "split %d of %d", i, n);
      next = r.end;
    }
    CHECK(next == s.tiles, "%d tiles in %d", s.tiles, n);
  }
}

int main() {
  for (uint32_t d = 1; d <= 70; ++d) check_div(d, 1);
  for (uint32_t d = 71; d <= (1u << 21); d = d * 9 / 8 + 1) check_div(d, 61);
  for (uint32_t s = 0; s <= 21; ++s)
    for (int e = -1; e <= 1; ++e)
      if ((int)(1u << s) + e >= 1) check_div((1u << s) + e, 97);
  for (int len : {0, 1, 7, 63, 64, 65, 130, 321, 700})
    for (int n : {1, 2, 5, 64, 100, 321})
      for (int window : {0, 1, 2, 63, 64, 65, 200, 1 << 23})
        for (int sinks : {0, 1, 4, 63, 64, 65, 130, 1 << 24})
          for (int split : {0, 1}) {
            const int place = len - n;  // may be negative: rows before the sequence
            const int first = split ? place + n / 2 : place;
            check_seen(first, len - 1, len, window, sinks);
            check_seen(first, first, len, window, sinks);
          }
  // whatever the arrays hold, rows stay in bounds
  for (int cu : {-2000000000, -1, 0, 3, 10, 11, 2000000000})
    for (int next : {-2000000000, 0, 3, 5, 10, 2000000000})
      for (int len : {-2147483647, -1, 0, 4, 5000, 2147483647})
        for (int most : {1, 4, 100}) {
          const NewTokens t = new_tokens(cu, next, len, 10, most, 4096);
          CHECK(t.first >= 0 && t.n >= 0 && t.n <= most && t.first + t.n <= 10, "%d %d", cu, next);
          CHECK(t.len >= 0 && t.len <= 4096 && t.place >= -10 && t.place <= 1 << 24, "%d", len);
        }
  const NewTokens t = new_tokens(3, 7, 100, 10, 4, 4096);
  CHECK(t.first == 3 && t.n == 4 && t.place == 96 && t.len == 100, "%d", t.place);
  std::printf("ok\n");
}
"""


def test_page_ranges_on_the_host(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "t")
    csrc = os.path.join(ROOT, "paper_2609_09208_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", csrc, "-o", exe, str(src)], check=True)
    got = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and got.stdout.strip() == "ok", got.stdout[-2000:]

"""The masks that the paged attention kernels apply to a tile's keys (csrc/page_ranges.hpp), compiled for the host, key by key:
together with the tiles that a row tile goes through, every key that the definition shows a query is seen once, and no other."""
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

// tokens p_first .. p_last of a row tile, keys 0 .. len - 1
static void check(int p_first, int p_last, int len, int window, int n_sink) {
  const SeenTiles s = seen_tiles(p_first, p_last, len, window, n_sink);
  for (int p = p_first; p <= p_last; p += p_last - p_first > 20 ? 13 : 1) {
    std::vector<int> in(len + 64, 0);
    for (int j = 0; j < s.tiles; ++j) {
      const int t0 = tile_start(s, j);
      if (whole_tile(s, p_first, p_last, t0, window, n_sink)) {
        for (int e = 0; e < kWTile; ++e) ++in[t0 + e];
        continue;
      }
      for (int at : {0, 8, 16, 24}) {  // a lane's first key, and its groups of 8 from there on
        const SeenKeys k = seen_keys(p, s.end, t0 + at, window, n_sink);
        for (int e0 : {0, 32}) {
          const uint32_t bits = seen_bits(k, e0);
          CHECK(bits <= 0xFFu, "%x", bits);
          for (int e = 0; e < 8; ++e) in[t0 + at + e0 + e] += (bits >> e) & 1;
        }
      }
    }
    for (int k = 0; k < len + 64; ++k) {
      const bool want = k < len && k <= p && (window <= 0 || k > p - window || k < n_sink);
      CHECK(in[k] == want, "place %d of %d..%d, %d keys, window %d, sinks %d: key %d %d times", p, p_first, p_last, len, window,
            n_sink, k, in[k]);
    }
  }
}

int main() {
  for (int len : {1, 7, 63, 64, 65, 100, 321, 700})
    for (int first : {-3, 0, 1, 50, 63, 64, 99, 190, 321, 400, 690, 999})
      for (int n : {1, 2, 40, 129})
        for (int window : {0, 1, 2, 50, 63, 64, 65, 200, 1000, (1 << 24) - 1})
          for (int sinks : {0, 1, 4, 63, 64, 65, 70, 130, 1 << 24}) check(first, first + n - 1, len, window, sinks);
  // the farthest places
  const int far = 1 << 24;
  for (int window : {0, 1, 64, far - 1})
    for (int sinks : {0, 3, far}) {
      const SeenKeys k = seen_keys(far - 1, far - 8, far - 64, window, sinks);
      for (int e0 : {0, 8, 48, 56})
        for (int e = 0; e < 8; ++e) {
          const int key = far - 64 + e0 + e;
          const bool want = key < far - 8 && (window == 0 || key > far - 1 - window || key < sinks);
          CHECK(((seen_bits(k, e0) >> e) & 1) == want, "key %d", key);
        }
    }
  std::printf("ok\n");
}
"""


def test_masks_and_tiles_are_the_definition(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "t")
    csrc = os.path.join(ROOT, "paper_2609_09208_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", csrc, "-o", exe, str(src)], check=True)
    got = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and got.stdout.strip() == "ok", got.stdout[-2000:]

"""How the row tiles of a paged attention call are split into pieces (csrc/page_ranges.hpp), compiled for the host: whatever
the sequences, every row tile has its pieces and they fit the launch, which holds one a row tile and `extra` more."""
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

struct Sequences {
  int count, fresh, len;  // `count` sequences of `fresh` new tokens and `len` in all
};

// G query heads a kv head, tiles of R rows, room for `extra` pieces more
static void check_call(const std::vector<Sequences>& all, int G, int R, int extra) {
  struct Shape { long long count; int rows, keys; };
  std::vector<Shape> shapes;
  long long tokens = 0, work = 0, row_tiles = 0, most_tiles = 0, longest = 1;
  for (const Sequences& s : all) {
    const int rows = (int)(((long long)s.fresh * G + R - 1) / R), last = (rows - 1) * R / G;
    const int seen = seen_tiles(s.len - s.fresh + last, s.len - 1, s.len, 0, 0).tiles;
    shapes.push_back({s.count, rows, seen < 1 ? 1 : seen});
    tokens += (long long)s.count * s.fresh;
    row_tiles += (long long)s.count * rows;
    work += (long long)s.count * rows * shapes.back().keys;
    most_tiles += s.count;
    if (shapes.back().keys > longest) longest = shapes.back().keys;
  }
  most_tiles += tokens * G / R;  // the launch's tiles
  int passes = 0;
  auto total_of = [&](int range) {
    ++passes;
    CHECK(range >= kManyRange && range <= kNoSplit, "range %d", range);
    long long n = 0;
    for (const Shape& s : shapes) {
      const int pieces = pieces_of(s.rows, s.keys, range);
      CHECK(pieces >= s.rows && pieces % s.rows == 0, "%d pieces of %d row tiles at %d", pieces, s.rows, range);
      n += s.count * pieces;
    }
    return (int64_t)n;
  };
  const PieceRange p = piece_range(extra, tokens * G / R, work, row_tiles, total_of);
  CHECK(p.total == total_of(p.range), "%lld", (long long)p.total);
  CHECK(p.total >= row_tiles && p.total <= row_tiles + extra && p.total <= most_tiles + extra,
        "%lld pieces of %lld row tiles, %d more", (long long)p.total, row_tiles, extra);
  if (extra == 0) CHECK(p.total == row_tiles, "%lld", (long long)p.total);
  if (row_tiles >= extra) CHECK(passes == 2, "%d passes", passes);  // one, and the check's own
  // many short tiles beside one that has more than the room's share of the work: it is split
  if (extra > 0 && longest > work / (extra / 2) && longest > kManyRange && row_tiles >= extra)
    CHECK(p.range < longest, "range %d of %lld tiles", p.range, longest);
}

int main() {
  check_call({{948, 17, 6720}}, 1, 256, 64);
  check_call({{1804, 3, 8960}}, 6, 256, 128);
  check_call({{1352, 3, 50304}}, 8, 256, 128);
  check_call({{1900, 17, 32768}, {1, 129, 32768}}, 1, 256, 128);
  check_call({{1600, 5, 131072}, {1, 40, 131072}}, 4, 256, 128);
  check_call({{2000, 17, 100}, {1, 200, 100000}}, 1, 256, 128);
  check_call({{1, 512, 8192}}, 8, 256, 128);
  check_call({{65535, 17, (1 << 24) - 8}}, 1, 256, 512);
  for (int hkv : {1, 2, 3, 8, 128})
    for (int G : {1, 4, 6, 8})
      for (int R : {128, 256})
        for (int count : {1, 2, 5, 60, 63, 64, 65, 130, 400, 511, 512, 513, 900, 3000, 65534})
          for (int fresh : {1, 17, 22, 100, 300})
            for (int len : {1, 64, 500, 513, 3000, 8960, 50304, 1 << 20, (1 << 24) - 8})
              for (int one : {0, 129, 5000}) {
                std::vector<Sequences> s = {{count, fresh, len}};
                if (one) s.push_back({1, one, 40000});
                const long long tokens = (long long)count * fresh + one;
                const bool split = (tokens * G + R - 1) / R * hkv < 512;
                check_call(s, G, R, split ? 512 / hkv : 0);
              }
  // any range that a piece can get covers a row tile's keys once
  for (int keys : {1, 7, 8, 9, 105, 4000, 1 << 18})
    for (int range : {8, 9, 100, 3000, 1 << 18, kNoSplit}) {
      const int n = pieces_of(1, keys, range);
      int next = 0;
      for (int i = 0; i < n; ++i) {
        const TileRun r = split_tiles(keys, i, n);
        CHECK(r.first == (next < keys ? next : keys) && r.end >= r.first, "%d", i);
        next = r.end;
      }
      CHECK(next == keys, "%d of %d", next, keys);
    }
  std::printf("ok\n");
}
"""


def test_pieces_cover_every_row_tile(tmp_path):
    src = tmp_path / "t.cpp"
    src.write_text(PROGRAM)
    exe = str(tmp_path / "t")
    csrc = os.path.join(ROOT, "paper_2609_09208_amd", "csrc")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", csrc, "-o", exe, str(src)], check=True)
    got = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and got.stdout.strip() == "ok", got.stdout[-2000:]

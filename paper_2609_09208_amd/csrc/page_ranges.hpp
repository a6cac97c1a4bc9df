// Arithmetic of paged caches and of what a query sees of one, plain enough for a host
// compiler: the tests check it there.
#pragma once

#include <stdint.h>

#include "key_ranges.hpp"

namespace potattn {

// Division of a group's number (8 tokens, below 2^21) by the groups of a page, as one high
// product: page = hi(2 group * mul) >> shift. With 2^shift <= d < 2^(shift + 1) and mul =
// ceil(2^(31 + shift) / d) <= 2^31 the excess 2 group (mul d - 2^(31 + shift)) stays below
// 2^22 d <= 2^(23 + shift) < 2^(32 + shift), so the quotient is exact.
struct PageDiv {
  uint32_t mul, shift;
};
POT_BOTH constexpr PageDiv page_div(uint32_t d) {
  uint32_t shift = 0;
  while ((d >> (shift + 1)) != 0) ++shift;
  return {(uint32_t)(((1ull << (31 + shift)) + d - 1) / d), shift};
}
POT_BOTH constexpr uint32_t page_of_group(uint32_t group, PageDiv v) {
  return (uint32_t)(((uint64_t)(2 * group) * v.mul) >> 32) >> v.shift;
}

// A sequence's new tokens in the packed rows and its length, taken into bounds whatever the
// arrays hold: rows first .. first + n - 1, the first of which is token `place` of the
// sequence (it may be negative: such a token sees nothing and is stored nowhere).
struct NewTokens {
  int first, n, place, len;
};
POT_BOTH constexpr NewTokens new_tokens(int cu, int cu_next, int len, int n_rows, int most_new,
                                        int most_len) {
  const int first = cu < 0 ? 0 : cu > n_rows ? n_rows : cu;
  const int end = cu_next < first ? first : cu_next > n_rows ? n_rows : cu_next;
  const int all = len < 0 ? 0 : len > (1 << 24) ? (1 << 24) : len;
  return {first, end - first < most_new ? end - first : most_new, all - (end - first),
          all < most_len ? all : most_len};
}

// The keys that tokens p_first .. p_last of a sequence of len keys see, as 64-key tiles in
// two runs: the sinks' (from key 0) and the window's (from key `low`, a multiple of 64). A
// token at place p sees key j if j <= p and (j > p - window or j < n_sink); window <= 0:
// every j <= p. Places may lie past the keys, and then so may the window.
struct SeenTiles {
  int sink_tiles;  // tiles 0 .. sink_tiles - 1 start at key 64 i
  int low;         // tile sink_tiles + i starts at key low + 64 i
  int tiles;       // of both runs
  int end;         // no key at or past it is seen
};
POT_BOTH constexpr SeenTiles seen_tiles(int p_first, int p_last, int len, int window, int n_sink) {
  const int end = p_last + 1 < len ? p_last + 1 : len;
  if (end <= 0) return {0, 0, 0, 0};
  int low = 0, sinks = 0;
  if (window > 0 && p_first >= window) {
    low = (p_first - window + 1) / kWTile * kWTile;
    sinks = (n_sink + kWTile - 1) / kWTile;
    if (n_sink <= 0) sinks = 0;
    if (sinks * kWTile >= low) {  // one run
      low = 0;
      sinks = 0;
    }
  }
  const int all = (end + kWTile - 1) / kWTile;  // tiles with keys
  if (sinks > all) sinks = all;
  return {sinks, low, sinks + (end > low ? all - low / kWTile : 0), end};
}
POT_BOTH constexpr int tile_start(const SeenTiles& s, int j) {
  return j < s.sink_tiles ? j * kWTile : s.low + (j - s.sink_tiles) * kWTile;
}
POT_BOTH constexpr bool sees(int p, int key, int window, int n_sink) {
  return key <= p && (window <= 0 || key > p - window || key < n_sink);
}
// Whether every token of p_first .. p_last (p_first >= 0) sees every key of t0 .. t0 + 63.
POT_BOTH constexpr bool all_seen(int p_first, int p_last, int t0, int window, int n_sink) {
  return t0 + kWTile - 1 <= p_first &&
         (window <= 0 || t0 > p_last - window || t0 + kWTile <= n_sink);
}
// The same where the keys may end before p_first.
POT_BOTH constexpr bool whole_tile(const SeenTiles& seen, int p_first, int p_last, int t0, int window,
                                   int n_sink) {
  return all_seen(p_first < seen.end ? p_first : seen.end - 1, p_last, t0, window, n_sink);
}
// Whether no token of them sees any.
POT_BOTH constexpr bool none_seen(int p_first, int p_last, int t0, int window, int n_sink) {
  return t0 > p_last || (window > 0 && t0 + kWTile - 1 <= p_first - window && t0 >= n_sink);
}

// Which of a tile's keys a query at `place` sees, t0 the tile's first, keys at or past `end` not there:
// key t0 + e is seen if e <= last and (e > before or e < sinks).
struct SeenKeys {
  int last, before, sinks;
};
POT_BOTH constexpr SeenKeys seen_keys(int place, int end, int t0, int window, int n_sink) {
  return {(place < end - 1 ? place : end - 1) - t0, window > 0 ? place - window - t0 : -1, n_sink - t0};
}
// The keys t0 + e0 .. t0 + e0 + 7 that it sees as bits.
POT_BOTH constexpr uint32_t first_bits(int n) {  // of 8
  return (1u << (n < 0 ? 0 : n > 8 ? 8 : n)) - 1u;
}
POT_BOTH constexpr uint32_t seen_bits(const SeenKeys& s, int e0) {
  return first_bits(s.last + 1 - e0) & (~first_bits(s.before + 1 - e0) | first_bits(s.sinks - e0)) & 0xFFu;
}

// Tiles j0 .. j1 - 1 of split i of n.
struct TileRun {
  int first, end;
};
POT_BOTH constexpr TileRun split_tiles(int tiles, int split, int n_splits) {
  const int per = (tiles + n_splits - 1) / n_splits;
  const int first = split * per < tiles ? split * per : tiles;
  return {first, first + per < tiles ? first + per : tiles};
}

// Key ranges of row tiles with many rows. A sequence of `rows` row tiles that see up to `keys` key tiles
// makes a piece for each row tile and range of `range` key tiles; the shortest range and the longest
// (of no split), in tiles.
constexpr int kManyRange = 8, kNoSplit = 1 << 24;
POT_BOTH constexpr int pieces_of(int rows, int keys, int range) {
  return rows * ((keys + range - 1) / range);
}
// The range for a call that may split its row tiles into `extra` pieces more (0: none), and the pieces of
// all sequences. work: the sequences' sum of rows * keys, row_tiles that of rows, call_tiles the row tiles
// that the call's rows make without a sequence's end; total_of(range): the sequences' sum of pieces_of.
// Half a piece a row tile is lost by rounding up, of as many as the call's rows make: the first range
// leaves room for that. Fewer row tiles than `extra` are then given wider ranges until there are at most
// `extra` pieces; more of them never are, and keep the range.
// There are at least row_tiles pieces and, with rows * (keys + range - 1) / range added up, at most
// row_tiles + work / range <= row_tiles + extra.
struct PieceRange {
  int range;
  int64_t total;
};
template <class Total>
POT_BOTH PieceRange piece_range(int extra, int64_t call_tiles, int64_t work, int64_t row_tiles,
                                Total total_of) {
  int64_t range = kNoSplit;
  if (extra > 0) {
    const int64_t most = extra - (call_tiles < extra ? call_tiles : extra) / 2;
    const int64_t even = (work + most - 1) / most;
    range = even < kManyRange ? kManyRange : even < kNoSplit ? even : kNoSplit;
  }
  int64_t total = total_of((int)range);
  for (int tries = 0; row_tiles < extra && total > extra && tries < 5; ++tries) {
    const int64_t wider = range * (total - extra) / extra;
    range += wider < 1 ? 1 : wider;
    if (range > kNoSplit) range = kNoSplit;
    total = total_of((int)range);
  }
  return {(int)range, total};
}

}  // namespace potattn
